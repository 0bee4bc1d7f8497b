"""Pages of the cache: fork, extend, free, compact, copy.  Oracle pins, refusals (CPU) and GPU parity, to the last integer."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ops
from paper_2603_06588_b200 import binding

from ._ops import FAKE_HANDLE, no_device, struct_fields


# --------------------------------------------------------------------------------------------------- CPU
@pytest.mark.parametrize("name,cls", [("hook_cache_pool", binding.HookCachePool), ("hook_cache_copy_params", binding.HookCacheCopyParams)])
def test_struct_mirror(name, cls):
    assert struct_fields(name) == [f[0] for f in cls._fields_]


def _consistent(pool):
    """Every page counts the table entries that name it."""
    refs = [0] * len(pool.refs)
    for row, L in zip(pool.table, pool.lens):
        held = row[:-(-L // 16)]
        assert all(p >= 0 for p in held) and all(p == -1 for p in row[len(held):])
        for p in held:
            refs[p] += 1
    assert refs == pool.refs


def test_oracle_life_cycle():
    pool = ops.Pool(4, 6, 12)
    assert pool.extend([20, 0, 0, 0]) == [(-1, -1)] * 4
    assert pool.table[0][:2] == [0, 1] and pool.refs[:3] == [1, 1, 0]
    pool.fork([0, 0], [1, 2])
    assert pool.refs[:2] == [3, 3] and pool.lens == [20, 20, 20, 0]
    pairs = pool.extend([0, 1, 13, 0])                           # both leave the shared page; the second needs another one too
    assert pairs == [(-1, -1), (1, 2), (1, 3), (-1, -1)]
    assert pool.table[1][:2] == [0, 2] and pool.table[2][:3] == [0, 3, 4] and pool.refs[:5] == [3, 1, 1, 1, 1]
    _consistent(pool)
    pool.free([0, 0, 2], [16, 0, 0])
    assert pool.lens == [16, 21, 0, 0] and pool.refs[:5] == [2, 0, 1, 0, 0]
    _consistent(pool)
    table, refs, page_map, moves = pool.compact()
    assert moves == [(2, 1)] and refs[:3] == [2, 1, 0] and table[1][:2] == [0, 1] and page_map[:3] == [0, -1, 1]
    assert not pool.faults


def test_oracle_copy():
    cache = np.arange(6)
    out, refused = ops.copy_pages(cache, [(0, 3), (0, 4), (-1, 2), (5, 5)])
    assert out.tolist() == [0, 1, 2, 0, 0, 5] and not refused
    assert ops.copy_pages(cache, [(0, 1), (1, 2)])[1] and ops.copy_pages(cache, [(0, 1), (2, 1)])[0].tolist() == cache.tolist()


def _pool_params(**over):
    p = binding.HookCachePool(4, 8, 64, 16, 0x10000, 0x20000, 0x30000, None)
    for k, v in over.items():
        setattr(p, k, v)
    return p


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), binding.HOOK_ATTN_ERR_CUDA), (dict(num_seqs=-1), binding.HOOK_ATTN_ERR_INVALID_ARG), (dict(block_table=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(seq_lens=None), binding.HOOK_ATTN_ERR_INVALID_ARG), (dict(page_refs=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(page_size=32), binding.HOOK_ATTN_ERR_UNSUPPORTED), (dict(num_seqs=16385), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(num_seqs=16384, max_blocks_per_seq=65537), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(num_blocks=2 ** 30 + 1), binding.HOOK_ATTN_ERR_UNSUPPORTED), (dict(num_blocks=2 ** 30), binding.HOOK_ATTN_ERR_CUDA), (dict(num_seqs=16384, max_blocks_per_seq=65536), binding.HOOK_ATTN_ERR_CUDA)])
def test_pool_refusals(over, code):
    lib, p = binding.load_library(), ctypes.byref(_pool_params(**over))
    assert lib.hook_cache_fork(FAKE_HANDLE, p, 0x1000, 0x1000, 1, None) == code
    assert lib.hook_cache_extend(FAKE_HANDLE, p, 0x1000, 0x1000, None) == code
    assert lib.hook_cache_free(FAKE_HANDLE, p, 0x1000, None, 1, None) == code
    assert lib.hook_cache_compact(FAKE_HANDLE, p, 0x1000, 0x2000, 0x3000, 0x4000, 0x5000, None) == code


@no_device
def test_list_refusals():
    lib, p, bad = binding.load_library(), ctypes.byref(_pool_params()), binding.HOOK_ATTN_ERR_INVALID_ARG
    assert lib.hook_cache_fork(FAKE_HANDLE, p, None, 0x1000, 1, None) == bad
    assert lib.hook_cache_fork(FAKE_HANDLE, p, 0x1000, 0x1000, -1, None) == bad
    assert lib.hook_cache_fork(FAKE_HANDLE, p, 0x1000, 0x1000, 16385, None) == binding.HOOK_ATTN_ERR_UNSUPPORTED
    assert lib.hook_cache_free(FAKE_HANDLE, p, 0x1000, None, 16385, None) == binding.HOOK_ATTN_ERR_UNSUPPORTED
    assert lib.hook_cache_extend(FAKE_HANDLE, p, 0x1000, None, None) == bad
    assert lib.hook_cache_free(FAKE_HANDLE, p, None, None, 1, None) == bad
    assert lib.hook_cache_compact(FAKE_HANDLE, p, 0x1000, 0x30000, 0x3000, 0x4000, 0x5000, None) == bad      # the counts in place
    assert lib.hook_cache_compact(FAKE_HANDLE, p, 0x1000, 0x2000, 0x30000, 0x4000, 0x5000, None) == bad
    assert lib.hook_cache_compact(FAKE_HANDLE, p, 0x1000, 0x2000, 0x3000, 0x4000, None, None) == bad
    assert lib.hook_cache_fork(FAKE_HANDLE, None, 0x1000, 0x1000, 1, None) == bad
    assert lib.hook_cache_fork(None, p, 0x1000, 0x1000, 1, None) == bad


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), binding.HOOK_ATTN_ERR_CUDA), (dict(num_layers=-1), binding.HOOK_ATTN_ERR_INVALID_ARG), (dict(pairs=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(k_caches=None), binding.HOOK_ATTN_ERR_INVALID_ARG), (dict(kv_block_stride=0), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(head_dim=80), binding.HOOK_ATTN_ERR_UNSUPPORTED), (dict(page_size=8), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(kv_head_stride=132), binding.HOOK_ATTN_ERR_UNSUPPORTED), (dict(address=0x10008), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(address=0), binding.HOOK_ATTN_ERR_INVALID_ARG), (dict(max_pairs=2 ** 30), binding.HOOK_ATTN_ERR_CUDA),
    (dict(max_pairs=2 ** 30 + 1), binding.HOOK_ATTN_ERR_UNSUPPORTED)])
def test_copy_refusals(over, code):
    at = over.pop("address", 0x10000) if "address" in over else 0x10000
    ptrs = (ctypes.c_void_p * 2)(0x10000, at)
    p = binding.HookCacheCopyParams(2, 64, 16, 8, 128, 4, 16 * 1024, 1024, 128, ctypes.addressof(ptrs), ctypes.addressof(ptrs), 0x20000, None, None)
    for k, v in over.items():
        setattr(p, k, v)
    assert binding.load_library().hook_cache_copy_pages(FAKE_HANDLE, ctypes.byref(p), None) == code


# --------------------------------------------------------------------------------------------------- GPU
@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


class Both:
    """The same pool on the device and as the oracle's lists."""

    def __init__(self, eng, num_seqs, max_blocks, num_blocks):
        self.eng, self.want = eng, ops.Pool(num_seqs, max_blocks, num_blocks)
        self.load()

    def load(self):
        t = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        w = self.want
        self.dev = dict(block_table=t(w.table).reshape(len(w.lens), w.max_blocks), seq_lens=t(w.lens), page_refs=t(w.refs),
                        status=torch.zeros(1, dtype=torch.int32, device="cuda"))

    def _i32(self, a):
        return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")

    def compare(self):
        torch.cuda.synchronize()
        assert self.dev["seq_lens"].tolist() == self.want.lens
        assert self.dev["page_refs"].tolist() == self.want.refs
        assert self.dev["block_table"].tolist() == self.want.table
        codes = {"bounds": binding.HOOK_ATTN_ERR_BOUNDS, "no pages": binding.HOOK_ATTN_ERR_NO_PAGES}
        assert int(self.dev["status"].item()) == min([codes[f] for f in self.want.faults], default=0)
        self.dev["status"].zero_()
        self.want.faults = []

    def fork(self, parents, children):
        self.eng.hook_cache_fork(**self.dev, parents=self._i32(parents), children=self._i32(children))
        self.want.fork(parents, children)
        self.compare()

    def extend(self, new_rows):
        pairs = self.eng.hook_cache_extend(**self.dev, new_rows=self._i32(new_rows))
        want = self.want.extend(new_rows)
        self.compare()
        assert [tuple(p) for p in pairs.tolist()] == want
        return want

    def free(self, seqs, keep=None):
        self.eng.hook_cache_free(**self.dev, seqs=self._i32(seqs), keep_lens=self._i32(keep))
        self.want.free(seqs, keep)
        self.compare()

    def compact(self, adopt=True):
        table, refs, page_map, pairs, count = self.eng.hook_cache_compact(**self.dev)
        want_table, want_refs, want_map, moves = self.want.compact()
        self.compare()                                            # the pool itself has not changed
        assert table.tolist() == want_table and refs.tolist() == want_refs and page_map.tolist() == want_map
        assert count.tolist() == [len(moves)]
        assert [tuple(p) for p in pairs.tolist()] == moves + [(-1, -1)] * (len(refs) // 2 - len(moves))
        if adopt:
            self.want.table, self.want.refs = want_table, want_refs
            self.load()


@pytest.mark.gpu
@pytest.mark.parametrize("num_blocks", [16383, 16385, 70001])
def test_large_pools(eng, num_blocks):
    """More pages than one step of a scan, most of them taken, so that the free ones lie far apart; and a view that no vector load may touch."""
    g = np.random.default_rng(num_blocks)
    both = Both(eng, 60, 2000, num_blocks)
    both.extend(g.integers(0, num_blocks * 16 // 60, 60).tolist())
    both.free(g.integers(0, 60, 30).tolist(), g.integers(0, num_blocks * 10 // 60, 30).tolist())
    both.fork([0, 1, 2], [57, 58, 59])
    both.extend(g.integers(0, 3000, 60).tolist())
    both.free([3, 9, 27, 31])
    both.dev["page_refs"] = torch.cat([both.dev["page_refs"][:1], both.dev["page_refs"]])[1:]
    both.compact(adopt=False)
    both.extend(g.integers(0, 500, 60).tolist())
    both.compact()


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("num_seqs,max_blocks,num_blocks", [(1, 1, 1), (3, 4, 7), (40, 9, 150), (300, 40, 3000), (1100, 5, 2500)])
def test_random_life(eng, seed, num_seqs, max_blocks, num_blocks):
    g = np.random.default_rng(seed)
    both = Both(eng, num_seqs, max_blocks, num_blocks)
    for _ in range(8):
        new = (g.integers(0, 40, num_seqs) * (g.random(num_seqs) < 0.6)).tolist()
        both.extend(new)
        n = int(g.integers(1, num_seqs + 1))
        both.fork(g.integers(0, num_seqs, n).tolist(), g.integers(0, num_seqs, n).tolist())
        both.extend((g.random(num_seqs) < 0.5).astype(int).tolist())
        both.free(g.integers(0, num_seqs, n // 2).tolist(), g.integers(0, 60, n // 2).tolist() if g.random() < 0.5 else None)
        if g.random() < 0.5:
            both.compact()
        _consistent(both.want)


@pytest.mark.gpu
def test_sharers_that_leave_a_page_together_give_it_back(eng):
    both = Both(eng, 3, 4, 10)
    both.extend([20, 0, 0])
    both.fork([0, 0], [1, 2])
    assert both.extend([1, 1, 1]) == [(1, 2), (1, 3), (1, 4)]
    assert both.want.refs[1] == 0
    assert both.extend([0, 0, 60 - 21]) == [(-1, -1)] * 3         # and it is taken again
    assert 1 in both.want.table[2]


@pytest.mark.gpu
def test_pool_runs_out(eng):
    both = Both(eng, 5, 8, 6)
    both.extend([30, 40, 3, 17, 0])                               # 2 + 3 pages, then one, then none for the fourth
    assert both.want.lens == [30, 40, 3, 0, 0]
    both.extend([2, 8, 5, 1, 0])                                  # room in the pages that are there
    both.extend([1, 0, 0, 0, 0])
    assert both.want.lens == [32, 48, 8, 0, 0]


@pytest.mark.gpu
def test_exact_fit_and_full_rows(eng):
    both = Both(eng, 2, 3, 6)
    both.extend([48, 48])
    both.extend([1, 0])                                           # beyond the table's row
    both.free([1], [17])
    both.extend([0, 31])
    assert both.want.lens == [48, 48]


@pytest.mark.gpu
@pytest.mark.parametrize("break_it", ["length", "negative length", "table", "refs"])
def test_broken_pools_are_reported(eng, break_it):
    both = Both(eng, 4, 4, 20)
    both.extend([20, 20, 20, 0])
    if break_it == "length":
        both.want.lens[1] = 65
    elif break_it == "negative length":
        both.want.lens[1] = -3
    elif break_it == "table":
        both.want.table[1][1] = 20
    else:
        both.want.refs[both.want.table[1][1]] = 0
    both.load()
    if break_it != "refs":
        both.fork([1], [3])
    both.extend([1, 1, 0, 0])
    both.extend([0, 0, -1, 5])
    both.free([1, 7, -1])
    both.free([2], [-1])


@pytest.mark.gpu
def test_lengths_up_to_the_last_integer(eng):
    """A table that could hold more tokens than an int32 counts: the sums must not wrap around."""
    lens, refs = torch.tensor([2 ** 31 - 10, 0], dtype=torch.int32, device="cuda"), torch.ones(4, dtype=torch.int32, device="cuda")
    table = torch.zeros((2, 2 ** 27 + 64), dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pairs = eng.hook_cache_extend(table, lens, refs, torch.tensor([100, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), status=status)
    assert pairs.tolist() == [[-1, -1]] * 2 and lens.tolist() == [2 ** 31 - 10, 0] and refs.tolist() == [1] * 4
    assert int(status.item()) == binding.HOOK_ATTN_ERR_NO_PAGES          # the second asks for all pages there could be; the first is out of range


@pytest.mark.gpu
def test_refused_forks(eng):
    both = Both(eng, 6, 4, 30)
    both.extend([20, 33, 0, 0, 0, 5])
    both.fork([0, 1, 0, 2, 0, 9, 1], [2, 2, 5, 3, 0, 4, -1])      # named twice, not empty, a child as a parent, itself, rows that are not there
    assert both.want.lens == [20, 33, 0, 0, 0, 5]                 # row 2 is a parent here: refused too
    both.fork([0, 1], [2, 2])
    assert both.want.lens[2] == 20
    both.fork([4], [3])                                           # an empty parent
    assert both.want.lens[3] == 0


@pytest.mark.gpu
def test_in_place_table_of_compact(eng):
    both = Both(eng, 3, 4, 20)
    both.extend([20, 40, 60])
    both.free([1])
    table, lens, counts, status = (both.dev[name] for name in ("block_table", "seq_lens", "page_refs", "status"))
    pool = ctypes.byref(binding.HookCachePool(3, 4, 20, 16, table.data_ptr(), lens.data_ptr(), counts.data_ptr(), status.data_ptr()))
    out = torch.empty(20 * 4, dtype=torch.int32, device="cuda")
    refs, page_map, pairs, count = out[:20], out[20:40], out[40:60], out[60:61]
    rc = eng._lib.hook_cache_compact(eng._h, pool, both.dev["block_table"].data_ptr(), refs.data_ptr(), page_map.data_ptr(), pairs.data_ptr(),
                                     count.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    want_table, want_refs, _, _ = both.want.compact()
    assert rc == 0 and both.dev["block_table"].tolist() == want_table and refs.tolist() == want_refs


@pytest.mark.gpu
@pytest.mark.parametrize("num_blocks", [1, 2, 1023, 1024, 1025, 4095, 4096, 4097, 8192, 8193, 12289])
@pytest.mark.parametrize("shape", ["all", "none", "low", "high", "odd", "one high", "one free", "below 0"])
def test_compact_at_the_edges(eng, num_blocks, shape):
    """Pools of whole and broken segments, with the count of used pages on and beside their edges, small and large tables, in place too."""
    used = {"all": lambda i: True, "none": lambda i: False, "low": lambda i: i < min(4096, num_blocks // 2), "high": lambda i: i >= num_blocks // 2,
            "odd": lambda i: i % 2, "one high": lambda i: i == num_blocks - 1, "one free": lambda i: i != num_blocks // 3, "below 0": lambda i: i % 3 == 0}[shape]
    both = Both(eng, 3, 6000, num_blocks)
    w = both.want
    w.refs = [1 + i % 5 if used(i) else (-2 if shape == "below 0" else 0) for i in range(num_blocks)]
    held = [i for i in range(num_blocks) if used(i)]
    g = np.random.default_rng(num_blocks)
    for s in (0, 2):
        mine = g.permutation(held)[:5990].tolist()
        w.table[s][:len(mine)] = mine
        w.lens[s] = 16 * len(mine) - (3 if mine else 0)
    both.load()
    both.compact(adopt=False)
    table = both.dev["block_table"]
    pool = ctypes.byref(binding.HookCachePool(3, 6000, num_blocks, 16, *(both.dev[n].data_ptr() for n in ("block_table", "seq_lens", "page_refs", "status"))))
    refs, page_map, pairs, count = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (num_blocks, num_blocks, num_blocks, 1))
    want_table, want_refs, want_map, moves = w.compact()
    assert eng._lib.hook_cache_compact(eng._h, pool, table.data_ptr(), refs.data_ptr(), page_map.data_ptr(), pairs.data_ptr(), count.data_ptr(),
                                       torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    assert table.tolist() == want_table and refs.tolist() == want_refs and page_map.tolist() == want_map and count.tolist() == [len(moves)]


@pytest.mark.gpu
@pytest.mark.parametrize("num_blocks", [20, 5000])
def test_compact_reports_tables_that_name_free_pages(eng, num_blocks):
    both = Both(eng, 3, 6, num_blocks)
    w = both.want
    w.refs = [int(i % 2) for i in range(num_blocks)]
    w.table[0][:4], w.lens[0] = [1, 0, num_blocks - 2, num_blocks - 1], 64     # a free page that is moved to, one that is not, and one beyond the pool
    w.table[1][:2], w.lens[1] = [num_blocks, -5], 20
    both.load()
    both.compact(adopt=False)


@pytest.mark.gpu
def test_extend_in_a_pool_of_many_million_pages(eng):
    """More steps than the counts that are made of them; the free pages far apart, among them the first and the last."""
    n, i32 = 17 * 2 ** 20 + 5, dict(dtype=torch.int32, device="cuda")
    at = [0, 5, 16383, 16384, 40000, 2 ** 20, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 70000, n - 2, n - 1]
    refs = torch.ones(n, **i32)
    refs[torch.tensor(at, device="cuda")] = 0
    table, lens, status = torch.full((5, 4), -1, **i32), torch.zeros(5, **i32), torch.zeros(1, **i32)
    pairs = eng.hook_cache_extend(table, lens, refs, torch.tensor([33, 16, 64, 1, 40], **i32), status=status)
    assert table.tolist() == [at[:3] + [-1], at[3:4] + [-1] * 3, at[4:8], at[8:9] + [-1] * 3, [-1] * 4]       # the last one finds two of three
    assert lens.tolist() == [33, 16, 64, 1, 0] and pairs.tolist() == [[-1, -1]] * 5 and int(status.item()) == binding.HOOK_ATTN_ERR_NO_PAGES
    assert int((refs == 0).sum()) == 2 and int(refs[n - 1]) == 0 and int(refs[n - 2]) == 0
    eng.hook_cache_extend(table, lens, refs, torch.tensor([15, 0, 0, 15, 32], **i32))
    assert table[4].tolist() == at[9:] + [-1] * 2 and lens.tolist() == [48, 16, 64, 16, 32] and int(refs.min()) == 1


def _cache(layout, pages, hkv, d, layers, seed):
    g = torch.Generator().manual_seed(seed)
    shape = {"contiguous": (layers, 2, pages, 16, hkv, d), "interleaved": (layers, pages, 2, 16, hkv, d), "heads first": (layers, 2, pages, hkv, 16, d),
             "padded": (layers, 2, pages, 16, hkv, d + 8)}[layout]
    return torch.randint(-2 ** 15, 2 ** 15, shape, generator=g, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)


def _layers(cache, layout, d):
    out = []
    for c in cache:
        k, v = (c[:, 0], c[:, 1]) if layout == "interleaved" else (c[0], c[1])
        if layout == "heads first":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        out.append((k[..., :d], v[..., :d]))
    return out


def _check_copy(eng, pairs, layout="contiguous", pages=40, hkv=3, d=64, layers=2, count=None, expect_status=0):
    host = _cache(layout, pages, hkv, d, layers, 3)
    dev, want = host.cuda(), host.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eng.hook_cache_copy_pages(_layers(dev, layout, d), torch.tensor(pairs, dtype=torch.int32, device="cuda").reshape(-1, 2),
                              num_pairs=None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda"), status=status)
    torch.cuda.synchronize()
    live = pairs if count is None else pairs[:max(0, count)]
    for k, v in _layers(want, layout, d):
        for t in (k, v):
            t.copy_(torch.from_numpy(ops.copy_pages(t.contiguous().view(torch.int16).numpy(), live)[0]).view(torch.bfloat16))
    assert torch.equal(dev.cpu().view(torch.int16), want.view(torch.int16))
    assert int(status.item()) == expect_status


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["contiguous", "interleaved", "heads first", "padded"])
@pytest.mark.parametrize("hkv,d,layers", [(1, 64, 1), (3, 64, 2), (8, 128, 3), (1, 128, 70)])
def test_copy(eng, layout, hkv, d, layers):
    _check_copy(eng, [(0, 20), (0, 21), (7, 39), (-1, -1), (5, -1), (-3, 6), (4, 4), (19, 22)], layout, hkv=hkv, d=d, layers=layers)


@pytest.mark.gpu
@pytest.mark.parametrize("count", [0, 1, 3, 9, -2])
def test_copy_counts_on_the_device(eng, count):
    _check_copy(eng, [(0, 20), (1, 21), (2, 22), (3, 23)], count=count)


@pytest.mark.gpu
@pytest.mark.parametrize("pairs", [[(0, 1), (2, 1)], [(0, 1), (1, 2)], [(0, 1), (1, 0)], [(0, 1), (0, 1), (3, 4)], [(0, 40)], [(40, 0)], [(5, 5), (0, 5)]])
def test_dependent_pairs_are_refused(eng, pairs):
    _check_copy(eng, pairs, expect_status=binding.HOOK_ATTN_ERR_BOUNDS)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [300, 2000, 5003])
def test_many_pairs(eng, n):
    g = np.random.default_rng(n)
    order = g.permutation(2 * n)
    pairs = [(int(order[g.integers(0, n)]), int(order[n + i])) for i in range(n)]
    _check_copy(eng, pairs, pages=2 * n, hkv=1, layers=1)
    _check_copy(eng, pairs, pages=2 * n, hkv=1, layers=2, count=n // 3)
    pairs[n // 2] = (pairs[n // 2][0], pairs[3][1])               # one destination twice: neither is carried out
    _check_copy(eng, pairs, pages=2 * n, hkv=1, layers=1, expect_status=binding.HOOK_ATTN_ERR_BOUNDS)


@pytest.mark.gpu
def test_nothing_to_do(eng):
    both = Both(eng, 2, 2, 4)
    both.fork([], [])
    both.free([])
    both.extend([0, 0])
    both.compact()
    _check_copy(eng, [])
    eng.hook_cache_copy_pages([], torch.zeros((1, 2), dtype=torch.int32, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("max_pairs,count", [(2048, 2048), (2048, 2047), (2049, 2049), (2049, 3), (2100, None), (9000, 2048), (9000, 8999), (9000, 0)])
@pytest.mark.parametrize("layers", [1, 3, 5])
def test_copy_of_many_pairs(eng, max_pairs, count, layers):
    """Long lists, of which few or all count, some of them dead, some that depend on one another."""
    pages, g = 20000, np.random.default_rng(max_pairs + layers)
    perm = g.permutation(pages)[:2 * max_pairs].reshape(max_pairs, 2)
    perm[g.integers(0, max_pairs, 7)] = -1
    a, b = max_pairs // 2, max_pairs // 3
    if count != 0:
        perm[a, 1] = perm[0, 0] = perm[b, 1] = 17                  # two with one destination, which is a third one's source
    cache = torch.randint(-2 ** 15, 2 ** 15, (layers, 2, pages, 16, 1, 64), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    cache = cache.to(torch.int16).cuda().view(torch.bfloat16)
    before, status = cache.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    pairs = torch.tensor(perm, dtype=torch.int32, device="cuda")
    eng.hook_cache_copy_pages([(c[0], c[1]) for c in cache], pairs, None if count is None else torch.tensor([count], dtype=torch.int32, device="cuda"), status=status)
    moved, refused = ops.copy_pages(np.arange(pages), [tuple(p) for p in perm[:max_pairs if count is None else count].tolist()])
    want = before.view(torch.int16)[:, :, torch.tensor(moved, device="cuda")]
    assert torch.equal(cache.view(torch.int16), want)
    assert int(status.item()) == (binding.HOOK_ATTN_ERR_BOUNDS if refused else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("num_blocks", [900, 5000, 20000, 70000])
def test_pools_in_a_graph_on_another_stream(eng, num_blocks):
    """All calls on a pool captured once and replayed, each replay on the state that the one before left."""
    both, g = Both(eng, 40, 400, num_blocks), np.random.default_rng(num_blocks)
    both.extend((g.integers(0, num_blocks * 8 // 40, 40) * (np.arange(40) < 35)).tolist())
    parents, children, seqs, keep = [0, 1, 2], [37, 38, 39], [5, 6, 37, 38, 39], [30, 7, 0, 0, 0]
    new = g.integers(0, 60, 40).tolist()
    args = [both._i32(x) for x in (parents, children, new, seqs, keep)]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        eng.hook_cache_fork(**both.dev, parents=args[0], children=args[1])
        pairs = eng.hook_cache_extend(**both.dev, new_rows=args[2])
        eng.hook_cache_free(**both.dev, seqs=args[3], keep_lens=args[4])
        table, refs, page_map, moves, count = eng.hook_cache_compact(**both.dev)
    for _ in range(3):
        graph.replay()
        both.want.fork(parents, children)
        want_pairs = both.want.extend(new)
        both.want.free(seqs, keep)
        want_table, want_refs, want_map, want_moves = both.want.compact()
        both.compare()
        assert [tuple(p) for p in pairs.tolist()] == want_pairs
        assert table.tolist() == want_table and refs.tolist() == want_refs and page_map.tolist() == want_map and count.tolist() == [len(want_moves)]
        assert [tuple(p) for p in moves.tolist()] == want_moves + [(-1, -1)] * (num_blocks // 2 - len(want_moves))


def test_oracle_forks_held_pages_alone():
    pool = ops.Pool(3, 2, 4)
    pool.extend([20, 0, 0])
    pool.refs[1] = 0
    pool.fork([0], [1])
    assert pool.faults == ["bounds"] and pool.lens == [20, 0, 0] and pool.refs == [1, 0, 0, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("count", [0, -2])
def test_pages_that_nobody_holds_are_not_forked(eng, count):
    """A fork would raise their count to 1, and parent and child would then append into one page that neither seems to share."""
    both = Both(eng, 7, 4, 30)
    both.extend([20, 33, 5, 0, 0, 0, 0])
    both.want.refs[both.want.table[0][1]] = count
    both.want.refs[both.want.table[2][0]] = count
    both.load()
    both.fork([0, 1, 0, 2], [3, 4, 5, 6])
    assert both.want.lens == [20, 33, 5, 0, 33, 0, 0]
    both.extend([0, 1, 0, 0, 1, 0, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("counted", [False, True])
def test_lists_longer_than_can_be_checked(eng, counted):
    """Refused as a whole: held against one another, 2^30 pairs would keep the device busy for days."""
    n, i32 = 2 ** 22 + 1, dict(dtype=torch.int32, device="cuda")
    cache = torch.ones((2, 4, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
    cache[:, 1] = 2.0
    before, status = cache.clone(), torch.zeros(1, **i32)
    pairs = torch.full((n, 2), -1, **i32)
    pairs[0] = torch.tensor([0, 1], **i32)
    eng.hook_cache_copy_pages([(cache[0], cache[1])], pairs, torch.tensor([n], **i32) if counted else None, status=status)
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS and torch.equal(cache, before)
    eng.hook_cache_copy_pages([(cache[0], cache[1])], pairs, torch.tensor([1], **i32), status=status.zero_())      # a long list of which little counts
    assert int(status.item()) == 0 and (cache[:, 1] == 1.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("count", [2 ** 16, 2 ** 16 + 1, 265001])
def test_copy_of_long_lists(eng, count):
    """On both sides of the length from which a unit has all slabs, with pairs that depend on one another."""
    pages, g = 2 * 265001 + 3, torch.Generator(device="cuda").manual_seed(count)
    pairs = torch.randperm(pages, generator=g, device="cuda")[:2 * 265001].reshape(-1, 2).int()
    pairs[5000, 1] = pairs[60000, 1]
    pairs[9, 0] = -1
    cache = torch.randint(-2 ** 15, 2 ** 15, (3, 2, pages, 16, 1, 64), generator=g, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    want, status = cache.clone().view(torch.int16), torch.zeros(1, dtype=torch.int32, device="cuda")
    eng.hook_cache_copy_pages([(c[0], c[1]) for c in cache], pairs, torch.tensor([count], dtype=torch.int32, device="cuda"), status=status)
    live = torch.ones(count, dtype=torch.bool, device="cuda")
    live[[9, 5000, 60000]] = False
    src, dst = pairs[:count][live].long().T
    for layer in want:
        layer[:, dst] = layer[:, src]
    assert torch.equal(cache.view(torch.int16), want) and int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS


@pytest.mark.gpu
@pytest.mark.parametrize("num_blocks", [800, 3000, 16000, 40000])
def test_as_many_sequences_as_a_pool_can_have(eng, num_blocks):
    """Lists of 16384 entries, and every size of the kernel that hands pages out beside the largest tables."""
    n, g = 16384, np.random.default_rng(num_blocks)
    both = Both(eng, n, 3, num_blocks)
    both.extend((g.integers(1, 33, n) * (np.arange(n) % 3 == 0)).tolist())
    both.fork((np.arange(n) // 3 * 3).tolist(), g.permutation(n).tolist())
    both.extend((g.random(n) < 0.3).astype(int).tolist())
    both.free(g.permutation(n).tolist(), g.integers(0, 40, n).tolist())
    both.extend(g.integers(0, 3, n).tolist())
    both.compact()


@pytest.mark.gpu
def test_pages_behind_the_first_4_gigabytes(eng):
    """Elements whose places do not fit 32 bits, in both caches of an interleaved pool."""
    pages = 2 ** 32 // (2 * 16 * 8 * 128) + 5
    cache = torch.zeros((pages, 2, 16, 8, 128), dtype=torch.bfloat16, device="cuda")
    cache[1], cache[pages - 1] = torch.randn(cache.shape[1:], device="cuda").bfloat16(), torch.randn(cache.shape[1:], device="cuda").bfloat16()
    first, last = cache[1].clone(), cache[pages - 1].clone()
    eng.hook_cache_copy_pages([(cache[:, 0], cache[:, 1])], torch.tensor([[1, pages - 2], [pages - 1, 2]], dtype=torch.int32, device="cuda"))
    for page, want in ((1, first), (2, last), (pages - 2, first), (pages - 1, last)):
        assert torch.equal(cache[page], want)
    cache[1:3], cache[pages - 2:] = 0, 0
    assert not cache.any()
