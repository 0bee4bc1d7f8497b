"""The cache held in 4 bits: oracle pins, refusals (CPU); the quantising append, the read-back and the page copies (GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2603_06588_b200 import binding

from ._ops import FAKE_HANDLE, no_device, struct_fields

SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


# --------------------------------------------------------------------------------------------------- CPU
def test_struct_mirrors():
    for name, mirror in (("hook_q4_cache", binding.HookQ4Cache), ("hook_q4_read_params", binding.HookQ4ReadParams),
                         ("hook_q4_copy_params", binding.HookQ4CopyParams)):
        assert struct_fields(name) == [f[0] for f in mirror._fields_]


def test_slab_bytes():
    for d, group in SHAPES:
        assert binding.q4_slab_bytes(d, group) == q4.slab_bytes(d, group)
    for d, group in ((64, 128), (128, 16), (96, 32), (256, 32), (128, 0), (128, -32)):
        with pytest.raises(binding.HookAttnError):
            binding.q4_slab_bytes(d, group)


def test_oracle_layout_is_a_permutation():
    for d, group in SHAPES:
        for place in (q4.place_k, q4.place_v):
            seen = {place(t, e, d) for t in range(16) for e in range(d)}
            assert len(seen) == 16 * d and all(0 <= b < 8 * d for b, _ in seen)


def test_oracle_quantises():
    codes, step, low = q4.quantise(np.arange(32.0)[None] / 2, 32)                 # 15.5 / 15 is 1.03125 in bf16
    assert float(step[0, 0]) == 1.03125 and float(low[0, 0]) == 0 and codes[0].tolist() == [round(i / 2 / 1.03125) for i in range(32)]
    codes, step, low = q4.quantise(np.full((1, 64), -3.0), 32)
    assert not codes.any() and not step.any() and (low == -3).all()
    codes, step, _ = q4.quantise(np.array([[0.0, 15.0, 0.5, 1.5, 2.5] + [0.0] * 27]), 32)       # halves go to even
    assert float(step[0, 0]) == 1.0 and codes[0, :5].tolist() == [0, 15, 0, 2, 2]
    assert np.isnan(q4.quantise(np.array([[np.inf] + [0.0] * 31]), 32)[1]).all()
    assert np.isnan(q4.quantise(np.array([[3.3e38, -3.3e38] + [0.0] * 30]), 32)[1]).all()       # the range overflows
    g = np.random.default_rng(0)
    x = q4.bf16(g.normal(size=(6, 64)))
    slab = np.full(q4.slab_bytes(64, 32), 0xA5, dtype=np.uint8)
    for t in range(3):
        q4.store(slab, t, x[2 * t], x[2 * t + 1], 32)
    for part, (code, step, low) in enumerate(q4.load(slab, 64, 32)):
        for t in range(3):
            c, s, l = q4.quantise(x[2 * t + part], 32)
            assert np.array_equal(code[t], c) and np.array_equal(step[t], np.repeat(s, 32)) and np.array_equal(low[t], np.repeat(l, 32))
            assert np.all(np.abs(code[t] * step[t] + low[t] - x[2 * t + part]) <= step[t] * (0.5 + 15 / 256))


def _cache(**over):
    c = binding.HookQ4Cache()
    c.pages, c.block_stride, c.head_stride, c.group = 0x10000, 8 * 2560, 2560, 32
    for k, v in over.items():
        setattr(c, k, v)
    return c


OK, INVALID, UNSUPPORTED = binding.HOOK_ATTN_ERR_CUDA, binding.HOOK_ATTN_ERR_INVALID_ARG, binding.HOOK_ATTN_ERR_UNSUPPORTED   # OK: no device
CACHE_FAULTS = [(dict(pages=None), INVALID), (dict(pages=0x10008), UNSUPPORTED), (dict(block_stride=0), INVALID), (dict(head_stride=-2560), INVALID),
                (dict(head_stride=2568), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(group=256), UNSUPPORTED), (dict(), OK)]


@no_device
@pytest.mark.parametrize("over,code", CACHE_FAULTS)
def test_refusals_of_the_cache(over, code):
    from .test_rope_append import _params as rope_params
    lib = binding.load_library()
    rope, read = rope_params(k_cache=None, v_cache=None, kv_head_stride=0), _read_params()
    assert lib.hook_rope_append_q4(FAKE_HANDLE, ctypes.byref(rope), ctypes.byref(_cache(**over)), None) == code
    assert lib.hook_cache_read_q4(FAKE_HANDLE, ctypes.byref(read), ctypes.byref(_cache(**over)), None) == code


def _read_params(**over):
    p = binding.HookQ4ReadParams()
    p.num_seqs, p.num_kv_heads, p.head_dim, p.page_size = 2, 8, 128, 16
    p.num_blocks, p.max_blocks_per_seq, p.to_num_blocks, p.to_max_blocks_per_seq = 64, 8, 32, 8
    p.block_table = p.seq_lens = p.to_table = 0x10000
    p.k_cache, p.v_cache = 0x20000, 0x30000
    p.kv_block_stride, p.kv_token_stride, p.kv_head_stride = 16 * 8 * 128, 8 * 128, 128
    for k, v in over.items():
        setattr(p, k, v)
    return p


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), OK), (dict(num_seqs=0), OK), (dict(num_seqs=-1), INVALID), (dict(head_dim=0), INVALID), (dict(head_dim=96), UNSUPPORTED),
    (dict(page_size=32), UNSUPPORTED), (dict(num_kv_heads=65), UNSUPPORTED), (dict(num_seqs=65536), UNSUPPORTED), (dict(seq_lens=None), INVALID),
    (dict(block_table=None), INVALID), (dict(to_table=None), INVALID), (dict(to_table=None, to_max_blocks_per_seq=0), OK), (dict(k_cache=None), INVALID),
    (dict(v_cache=0x30008), UNSUPPORTED), (dict(kv_token_stride=0), INVALID), (dict(kv_token_stride=1028), UNSUPPORTED)])
def test_refusals_of_the_read_back(over, code):
    assert binding.load_library().hook_cache_read_q4(FAKE_HANDLE, ctypes.byref(_read_params(**over)), ctypes.byref(_cache()), None) == code


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), OK), (dict(max_pairs=0), OK), (dict(max_pairs=-1), INVALID), (dict(pairs=None), INVALID), (dict(group=16), UNSUPPORTED),
    (dict(head_dim=64, group=128), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(num_kv_heads=65), UNSUPPORTED), (dict(block_stride=0), INVALID),
    (dict(head_stride=2568), UNSUPPORTED), (dict(max_pairs=2 ** 30 + 1), UNSUPPORTED), (dict(pages=None), INVALID)])
def test_refusals_of_the_copy(over, code):
    p = binding.HookQ4CopyParams()
    p.num_layers, p.num_blocks, p.page_size, p.num_kv_heads, p.head_dim, p.group, p.max_pairs = 2, 64, 16, 8, 128, 32, 4
    p.block_stride, p.head_stride, p.pairs = 8 * 2560, 2560, 0x10000
    layers = (ctypes.c_void_p * 2)(0x10000, 0x20000)
    p.pages = ctypes.cast(layers, ctypes.c_void_p)
    for k, v in over.items():
        setattr(p, k, v)
    lib = binding.load_library()
    assert lib.hook_cache_copy_pages_q4(FAKE_HANDLE, ctypes.byref(p), None) == code
    layers[1] = 0x20008
    assert lib.hook_cache_copy_pages_q4(FAKE_HANDLE, ctypes.byref(p), None) == (UNSUPPORTED if code == OK and p.max_pairs else code)


def test_missing_arguments():
    lib = binding.load_library()
    for fn in (lib.hook_rope_append_q4, lib.hook_cache_read_q4):
        assert fn(None, None, None, None) == INVALID
        assert fn(None, None, ctypes.byref(_cache()), None) == INVALID
    assert lib.hook_cache_read_q4(None, ctypes.byref(_read_params()), None, None) == INVALID
    assert lib.hook_cache_read_q4(None, ctypes.byref(_read_params()), ctypes.byref(_cache()), None) == INVALID      # no handle
    assert lib.hook_cache_copy_pages_q4(None, None, None) == INVALID


# --------------------------------------------------------------------------------------------------- GPU
@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _paged(q_lens, ctx, seed, extra=3):
    """Lengths and a block table over shuffled pages."""
    g = np.random.default_rng(seed)
    lens = [c + n for c, n in zip(ctx, q_lens)]
    pages = [-(-L // 16) for L in lens]
    order = g.permutation(sum(pages) + extra).tolist()
    table = np.full((len(lens), max(pages + [1]) + 1), -1, dtype=np.int64)
    for s, n in enumerate(pages):
        table[s, :n], order = order[:n], order[n:]
    return lens, table, sum(pages) + extra


def _append(eng, k, v, pages, lens, table, cu, freq=(), q=None, **kw):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(k.shape[0], k.shape[1], k.shape[2], dtype=k.dtype, device="cuda") if q is None else q
    out = eng.hook_rope_append_q4(q=q, k=k, v=v, pages=pages, block_table=_i32(table), seq_lens=_i32(lens), cu_q_lens=None if cu is None else _i32(cu),
                                  inv_freq=torch.tensor(freq, dtype=torch.float32, device="cuda"), status=status, **kw)
    torch.cuda.synchronize()
    return out, int(status.item())


def _bytes_after(pages, k, v, lens, table, cu, group):
    """What the pages hold once rows ``k``, ``v`` (float64 of bf16 values, [T, Hkv, D]) are stored."""
    want = pages.copy()
    for s, L in enumerate(lens):
        n = cu[s + 1] - cu[s]
        for i in range(n):
            pos = L - n + i
            for h in range(k.shape[1]):
                q4.store(want[table[s, pos // 16], h], pos % 16, k[cu[s] + i, h], v[cu[s] + i, h], group)
    return want


def _rows(rows, hkv, d, dtype, seed, kind="normal"):
    g = np.random.default_rng(seed)
    x = g.normal(size=(2, rows, hkv, d))
    if kind == "scales":                                   # groups of very different sizes, constant ones and offsets
        x = x * 2.0 ** g.integers(-30, 30, size=(2, rows, hkv, 1)) + 2.0 ** g.integers(-30, 12, size=(2, rows, hkv, 1))
        x[:, ::5] = x[:, ::5, :, :1]
    elif kind == "grid":                                   # quotients that fall on halves
        x = np.round(x * 4) / 4
        x[..., 0], x[..., 1] = -7.5, 7.5
    return torch.from_numpy(x).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("dtype,kind", [(t, kind) for t in (torch.bfloat16, torch.float16, torch.float32) for kind in ("normal", "scales", "grid")
                                        if not (t == torch.float16 and kind == "scales")])         # fp16 does not reach those sizes
def test_append_writes_the_oracles_bytes(eng, d, group, dtype, kind):
    q_lens, ctx, hkv = [1, 0, 17, 3, 33], [15, 4, 0, 30, 7], 3
    lens, table, pool = _paged(q_lens, ctx, 2)
    cu = [0] + np.cumsum(q_lens).tolist()
    x = _rows(cu[-1], hkv, d, dtype, 3, kind)
    pages = np.random.default_rng(4).integers(0, 256, (pool, hkv, q4.slab_bytes(d, group)), dtype=np.uint8)
    dev = torch.from_numpy(pages).cuda()
    _, status = _append(eng, x[0].cuda(), x[1].cuda(), dev, lens, table, cu)
    want = _bytes_after(pages, x[0].to(torch.bfloat16).double().numpy(), x[1].to(torch.bfloat16).double().numpy(), lens, table, cu, group)
    assert status == 0 and np.array_equal(dev.cpu().numpy(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("d,group,rot,adjacent", [(128, 32, 128, False), (128, 128, 54, True), (64, 64, 40, False), (64, 32, 2, True), (128, 64, 90, False)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotated_keys_are_those_of_the_bf16_cache(eng, d, group, rot, adjacent, dtype):
    """Queries, and what is quantised, bit for bit as hook_rope_append leaves them; slices of one projection."""
    q_lens, ctx, hq, hkv = [5, 40, 1], [3, 0, 100], 6, 2
    lens, table, pool = _paged(q_lens, ctx, 5)
    cu = [0] + np.cumsum(q_lens).tolist()
    g = torch.Generator().manual_seed(6)
    qkv = torch.randn(cu[-1], hq + 2 * hkv, d, generator=g).to(dtype).cuda()
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    freq = (10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))).astype(np.float32).tolist()
    kw = dict(pairing=binding.HOOK_ROPE_PAIR_ADJACENT if adjacent else binding.HOOK_ROPE_PAIR_HALVES, factor=1.25)
    cache = torch.zeros(2, pool, 16, hkv, d, dtype=torch.bfloat16, device="cuda")
    want_q = eng.hook_rope_append(q=q, k=k, v=v, k_cache=cache[0], v_cache=cache[1], block_table=_i32(table), seq_lens=_i32(lens), cu_q_lens=_i32(cu),
                                  inv_freq=torch.tensor(freq, device="cuda"), **kw)
    pages = torch.zeros(pool, hkv, q4.slab_bytes(d, group), dtype=torch.uint8, device="cuda")
    got_q, status = _append(eng, k, v, pages, lens, table, cu, freq, q=q, **kw)
    assert status == 0 and torch.equal(got_q, want_q)
    at = [(int(table[s, p // 16]), p % 16) for s, L in enumerate(lens) for p in range(L - q_lens[s], L)]
    k2, v2 = (np.stack([cache[i, page, slot].double().cpu().numpy() for page, slot in at]) for i in (0, 1))
    want = _bytes_after(np.zeros(pages.shape, dtype=np.uint8), k2, v2, lens, table, cu, group)
    assert np.array_equal(pages.cpu().numpy(), want)


@pytest.mark.gpu
def test_append_of_values_that_are_not_finite(eng):
    """A group with an infinity, a NaN or too wide a range reads as NaN, its neighbours do not."""
    x = _rows(4, 1, 128, torch.bfloat16, 7)
    x[0, 0, 0, 40], x[0, 1, 0, 0], x[1, 2, 0, 127] = float("inf"), float("nan"), float("-inf")
    x[0, 3, 0, 64], x[0, 3, 0, 65] = 3.3e38, -3.3e38
    x[1, 3, 0, :32] = torch.tensor([0.0, 1e-38] * 16).to(torch.bfloat16)          # a range that counts as none
    pages = torch.zeros(1, 1, q4.slab_bytes(128, 32), dtype=torch.uint8, device="cuda")
    _, status = _append(eng, x[0].cuda(), x[1].cuda(), pages, [4], [[0]], [0, 4])
    kc, vc = (torch.zeros(1, 16, 1, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    eng.hook_cache_read_q4(pages, _i32([[0]]), _i32([4]), k_cache=kc, v_cache=vc, to_table=_i32([[0]]))
    k, v = kc[0, :4, 0].cpu(), vc[0, :4, 0].cpu()
    bad_k, bad_v = torch.zeros(4, 128, dtype=torch.bool), torch.zeros(4, 128, dtype=torch.bool)
    bad_k[0, 32:64] = bad_k[1, :32] = bad_k[3, 64:96] = bad_v[2, 96:] = True
    assert status == 0 and torch.equal(torch.isnan(k), bad_k) and torch.equal(torch.isnan(v), bad_v)
    assert not v[3, :32].any()


@pytest.mark.gpu
def test_append_refuses_rows_and_leaves_the_rest(eng):
    """Bad lengths and pages set status and zero their queries; rows behind the last sequence stay as they were; strided heads."""
    d, group, hkv = 64, 32, 2
    lens, cu = [3, 40, 2, 5, 20], [0, 1, 2, 5, 6, 7]                  # the third has more rows than tokens, the last two tables are bad
    table = np.array([[1, -1, -1], [2, 3, 4], [5, -1, -1], [-1, -1, -1], [6, 99, -1]])
    x = _rows(9, hkv, d, torch.bfloat16, 8).cuda()
    wide = torch.zeros(hkv, 8, q4.slab_bytes(d, group) + 16, dtype=torch.uint8, device="cuda")
    pages = wide.transpose(0, 1)[:, :, :-16]
    q_out = torch.full((9, hkv, d), 5.0, dtype=torch.bfloat16, device="cuda")
    q, status = _append(eng, x[0], x[1], pages, lens, table, cu, q=x[0], q_out=q_out)
    assert status == binding.HOOK_ATTN_ERR_BOUNDS
    assert torch.equal(q[[0, 1]], x[0][[0, 1]]) and not q[2:7].any() and (q[7:] == 5).all()
    rows = x.double().cpu().numpy()
    want = np.zeros((8, hkv, q4.slab_bytes(d, group)), dtype=np.uint8)
    for h in range(hkv):
        q4.store(want[1, h], 2, rows[0, 0, h], rows[1, 0, h], group)
        q4.store(want[4, h], 7, rows[0, 1, h], rows[1, 1, h], group)
    assert np.array_equal(pages.cpu().numpy(), want) and not wide[:, :, -16:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("hkv,hq,d,rows", [(1, 1, 64, 1), (64, 64, 128, 3), (8, 8, 128, 700), (5, 5, 64, 130)])
def test_append_at_the_sizes_of_a_decode_batch(eng, hkv, hq, d, rows):
    """One row for each sequence, unaligned rows of all heads included."""
    lens = (np.arange(rows) % 50 + 1).tolist()
    table = np.arange(rows * 4).reshape(rows, 4)
    flat = torch.from_numpy(np.random.default_rng(9).normal(size=2 * rows * hkv * d + 1)).to(torch.bfloat16).cuda()[1:].view(2, rows, hkv, d)
    pages = torch.zeros(rows * 4, hkv, q4.slab_bytes(d, 32), dtype=torch.uint8, device="cuda")
    _, status = _append(eng, flat[0], flat[1], pages, lens, table, None)
    kc, vc = (torch.zeros(rows * 4, 16, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    first = [L - 1 for L in lens]
    eng.hook_cache_read_q4(pages, _i32(table), _i32(lens), k_cache=kc, v_cache=vc, to_table=_i32(table), first=_i32(first))
    at = torch.tensor([table[r, p // 16] * 16 + p % 16 for r, p in enumerate(first)], device="cuda")
    assert status == 0
    for got, x in ((kc, flat[0]), (vc, flat[1])):
        got = got.flatten(0, 1)
        g = x.double().unflatten(2, (-1, 32))
        step = (g.amax(-1) - g.amin(-1)) / 15 * (1 + 2.0 ** -8)
        # half a step, what a step rounded down leaves out at the top (15 x 2^-8 of one), and the rounding of the read
        bound = step * (0.5 + 15 / 256) + g.abs().amax(-1) * 2.0 ** -8
        assert ((got[at].double().unflatten(2, (-1, 32)) - g).abs() <= bound[..., None]).all()
        got[at] = 0
        assert not got.any()                               # nothing else was read


@pytest.mark.gpu
@pytest.mark.parametrize("d,group", SHAPES)
def test_read_back(eng, d, group):
    """lowest + step * code to the nearest bf16, from `first` on; slots behind the sequence and pages in nobody's table stay."""
    lens, table, pool = _paged([0] * 6, [1, 16, 0, 100, 47, 33], 10)
    hkv = 3
    g = np.random.default_rng(11)
    slabs = g.integers(0, 256, (pool, hkv, q4.slab_bytes(d, group)), dtype=np.uint8)
    params = torch.from_numpy(g.normal(size=(pool, hkv, 64 * (d // group)))).to(torch.bfloat16).view(torch.uint8).numpy()
    slabs[..., 16 * d:] = params
    first = [0, 3, 0, 50, 48, 32]                          # one of them behind its sequence's end
    to = table[:, ::-1].copy()
    for s, L in enumerate(lens):
        n = -(-L // 16)
        to[s] = -1
        to[s, :n] = np.sort(table[s, :n])
    cache = torch.full((2, pool, 16, hkv, d + 8), 9.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eng.hook_cache_read_q4(torch.from_numpy(slabs).cuda(), _i32(table), _i32(lens), k_cache=cache[0, ..., :d], v_cache=cache[1, ..., :d], to_table=_i32(to),
                           first=_i32(first), status=status)
    want = np.full((2, pool, 16, hkv, d + 8), 9.0)
    for part, (code, step, low) in enumerate(q4.load(slabs, d, group)):
        value = (code * step + low).astype(np.float32)     # at most 4 + 8 bits next to 8: one rounding to 32 bits, then one to 16
        for s, L in enumerate(lens):
            for p in range(first[s], L):
                want[part, to[s, p // 16], p % 16, :, :d] = q4.bf16(value[table[s, p // 16], :, p % 16])
    assert int(status.item()) == 0 and np.array_equal(cache.double().cpu().numpy(), want)


@pytest.mark.gpu
def test_read_back_faults(eng):
    d, group = 64, 64
    pages = torch.zeros(4, 1, q4.slab_bytes(d, group), dtype=torch.uint8, device="cuda")
    pages[:, :, 16 * d:] = torch.tensor([0.0, 1.0], dtype=torch.bfloat16, device="cuda").view(torch.uint8).repeat(32)      # every element is 1
    for lens, table, to, first, filled in (([20], [[0, 9]], [[1, 2]], None, [1]), ([20], [[0, 1]], [[3, -1]], None, [3]), ([33], [[0, 1]], [[1, 2]], None, []),
                                           ([-1], [[0, 1]], [[1, 2]], None, []), ([20], [[0, 1]], [[1]], None, []), ([20], [[0, 1]], [[1, 2]], [-1], [])):
        kc, vc = (torch.zeros(4, 16, 1, d, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        eng.hook_cache_read_q4(pages, _i32(table), _i32(lens), k_cache=kc, v_cache=vc, to_table=_i32(to), first=None if first is None else _i32(first),
                               status=status)
        assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS
        assert [p for p in range(4) if kc[p].any() or vc[p].any()] == filled


@pytest.mark.gpu
@pytest.mark.parametrize("d,group,hkv,layers,wide", [(128, 32, 8, 3, False), (64, 64, 1, 131, False), (64, 32, 5, 2, True), (128, 128, 3, 1, True)])
def test_page_copies(eng, d, group, hkv, layers, wide):
    g = torch.Generator().manual_seed(12)
    pool, slab = 40, q4.slab_bytes(d, group)
    full = torch.randint(0, 256, (layers, pool, hkv, slab + 48 * wide), generator=g, dtype=torch.uint8)
    pairs = torch.randperm(pool, generator=g)[:24].view(12, 2).int()
    pairs[3], pairs[7, 0] = -1, pairs[2, 0]                # nothing to copy; one source twice
    dev = full.cuda()
    caches = [c[..., :slab] for c in dev]
    for count in (5, 12):
        eng.hook_cache_copy_pages_q4(caches, pairs.cuda(), num_pairs=_i32([count]))
        for a, b in pairs[:count].tolist():
            if a >= 0:
                full[:, b, :, :slab] = full[:, a, :, :slab]
        assert torch.equal(dev.cpu(), full)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    eng.hook_cache_copy_pages_q4(caches, _i32([[0, pool], [1, 2], [2, 3]]), status=status)     # outside the pool; a destination that is a source
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS and torch.equal(dev.cpu(), full)
    eng.hook_cache_copy_pages_q4([], _i32([[0, 1]]))


@pytest.mark.gpu
def test_refused_tensors(eng):
    """Checks of the binding: types, shapes, strides and devices of the pages."""
    pages = torch.zeros(4, 2, q4.slab_bytes(64, 32), dtype=torch.uint8, device="cuda")
    kc = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    table, lens, freq = _i32([[0]]), _i32([1]), torch.zeros(0, device="cuda")
    good = dict(k_cache=kc, v_cache=kc.clone(), to_table=table)
    eng.hook_cache_read_q4(pages, table, lens, **good)
    for bad in (pages[..., :-1], pages.int(), pages[:, :1], pages.cpu(), torch.zeros(4, 2, 2 * pages.shape[2], dtype=torch.uint8, device="cuda")[..., ::2]):
        with pytest.raises(AssertionError):
            eng.hook_cache_read_q4(bad, table, lens, **good)
        with pytest.raises(AssertionError):
            eng.hook_rope_append_q4(q=x, k=x, v=x, pages=bad, block_table=table, seq_lens=lens, inv_freq=freq)
    for bad in ([pages, pages[:2]], [pages.int()], [pages[..., :-16]], [None]):
        with pytest.raises(AssertionError):
            eng.hook_cache_copy_pages_q4(bad, _i32([[0, 1]]))
