"""The hooked attention over a 4-bit cache: refusals (CPU) and GPU parity with 64-bit sums over what the pages stand for."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2603_06588_b200 import binding

from ._ops import FAKE_HANDLE, no_device
from .test_q4_cache import CACHE_FAULTS, INVALID, OK, UNSUPPORTED, _cache, _i32


def bounds(size, out, q_dim):
    """What rounding may come to, of the output and of a span mass.  x: the scores are sums of q_dim products and a few more in 32 bits, each
    term at most size.x in all, on either side of the largest (2^-24 each, doubled for the matrix unit's alignment), and the
    exponentials are off by 2^-22; a probability errs by that, of itself.  The output adds: probabilities times steps rounded to halves (2^-11, and
    2^-25 of the steps' power of two for those below 2^-14 of it, for each of the keys and codes up to 15), 32-bit sums over
    the keys in pieces, and its rounding to bf16 (2^-8)."""
    p = 2 * size["x"] * (q_dim + 8) * 2.0 ** -23 + 2.0 ** -21
    sums = 2.0 ** -22 * 64 * size["largest"]
    return (np.abs(out) * 2.0 ** -8 + size["coded"] * 2.0 ** -11 + size["keys"] * 15 * size["step"] * 2.0 ** -25 + 2 * p * size["largest"] + sums, 2 * p + 2.0 ** -18)


# --------------------------------------------------------------------------------------------------- CPU
def _params(**over):
    p = binding.HookAttnParams()
    p.num_seqs = p.total_q = 2
    p.num_q_heads, p.num_kv_heads, p.head_dim, p.page_size, p.num_blocks, p.max_blocks_per_seq = 32, 8, 128, 16, 64, 8
    p.q, p.out, p.block_table, p.seq_lens = 0x10000, 0x20000, 0x30000, 0x40000
    p.workspace, p.workspace_bytes = 0x100000, 1 << 30
    for k, v in over.items():
        setattr(p, k, v)
    return p


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), OK), (dict(num_seqs=0, total_q=0), OK), (dict(total_q=3), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(seq_lens=None), INVALID), (dict(max_blocks_per_seq=0), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(num_q_heads=72), UNSUPPORTED),
    (dict(num_q_heads=30), INVALID), (dict(page_size=32), UNSUPPORTED), (dict(q=0x10008), UNSUPPORTED), (dict(num_spans=9), UNSUPPORTED),
    (dict(num_kv_heads=2), UNSUPPORTED), (dict(num_seqs=65536, total_q=65536), UNSUPPORTED),
    (dict(workspace=None), binding.HOOK_ATTN_ERR_WORKSPACE), (dict(workspace=0x100010), binding.HOOK_ATTN_ERR_WORKSPACE),
    (dict(workspace_bytes=4096), binding.HOOK_ATTN_ERR_WORKSPACE)])
def test_refusals(over, code):
    assert binding.load_library().hook_attn_decode_q4(FAKE_HANDLE, ctypes.byref(_params(**over)), ctypes.byref(_cache()), None) == code


@no_device
@pytest.mark.parametrize("over,code", CACHE_FAULTS)
def test_refusals_of_the_cache(over, code):
    assert binding.load_library().hook_attn_decode_q4(FAKE_HANDLE, ctypes.byref(_params()), ctypes.byref(_cache(**over)), None) == code


def test_missing_arguments_and_workspace():
    lib = binding.load_library()
    assert lib.hook_attn_decode_q4(None, None, ctypes.byref(_cache()), None) == INVALID
    assert lib.hook_attn_decode_q4(None, ctypes.byref(_params()), None, None) == INVALID
    assert lib.hook_attn_decode_q4(None, ctypes.byref(_params()), ctypes.byref(_cache()), None) == INVALID       # no handle
    size = lambda **over: int(lib.hook_attn_workspace_bytes(ctypes.byref(_params(**over)), 3))
    assert size() > 0 and size(head_dim=96) == 0
    many = dict(num_seqs=256, total_q=256, max_blocks_per_seq=512)
    assert size(**many, max_seq_len=300) < size(**many)


# --------------------------------------------------------------------------------------------------- GPU
@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _slabs(g, shape, d, group, kind="normal"):
    """Pages of random codes; steps and lowest values of a unit normal distribution, or of very different sizes."""
    slabs = g.integers(0, 256, (*shape, q4.slab_bytes(d, group)), dtype=np.uint8)
    n = 32 * (d // group)
    step, low = 0.2 + 0.1 * g.random((*shape, n)), -2.5 + g.random((*shape, n))
    if kind == "steps":                                    # V's from 2^-40 to 2^3, some 0
        size = 2.0 ** g.integers(-40, 4, size=(*shape, n // 2)) * (g.random((*shape, n // 2)) < 0.9)
        step[..., n // 2:] *= size
        low[..., n // 2:] *= size
    elif kind == "constant":
        step[:] = 0
    elif kind == "large":
        step *= 1000
        low *= 1000
    slabs[..., 16 * d:] = torch.from_numpy(np.stack([step, low], -1)).to(torch.bfloat16).view(torch.uint8).flatten(-2).numpy()
    return slabs


class Case:
    def __init__(self, lens, hq, hkv, d, group, seed=1, kind="normal", spans=0, steer=False, q_size=1.0, layout="tight", scale=0.0, width=0):
        g = np.random.default_rng(seed)
        self.lens, self.hq, self.hkv, self.d, self.group = lens, hq, hkv, d, group
        pages = [-(-max(L, 0) // 16) for L in lens]
        pool = sum(pages) + 2
        order = g.permutation(pool).tolist()
        self.table = np.full((len(lens), max([width, max(pages + [1]) + 2])), -1, dtype=np.int64)
        self.slabs = _slabs(g, (pool, hkv), d, group, kind)
        for s, n in enumerate(pages):
            self.table[s, :n], order = order[:n], order[n:]
        poison = self.slabs.copy()                         # NaN pairs in the slots and pages that no sequence has
        pairs = poison[..., 16 * d:].reshape(pool, hkv, 2, 16, -1)
        used = np.zeros((pool, 16), dtype=bool)
        for s, L in enumerate(lens):
            for p in range(max(L, 0)):
                used[self.table[s, p // 16], p % 16] = True
        pairs[:] = np.where(used[:, None, None, :, None], pairs, 255)
        poison[..., 16 * d:] = pairs.reshape(pool, hkv, -1)
        nbytes = self.slabs.shape[-1]
        if layout == "tight":
            self.pages = torch.from_numpy(poison).cuda()
        else:                                              # heads first, with room between the slabs
            wide = torch.zeros(hkv, pool, nbytes + 32, dtype=torch.uint8, device="cuda")
            self.pages = wide.transpose(0, 1)[..., :nbytes]
            self.pages.copy_(torch.from_numpy(poison))
        self.q = torch.from_numpy(g.normal(size=(len(lens), hq, d)) * q_size).to(torch.bfloat16)
        self.scale = scale
        self.spans = self.mask = self.alpha = self.steer = None
        if spans:
            at = g.integers(-5, max(max(lens), 1) + 20, size=(len(lens), spans, 2))
            self.spans = torch.from_numpy(np.sort(at, -1)).int()
            self.spans[:, 0] = torch.tensor([0, 1 << 30])
            self.mask = torch.from_numpy((g.random(hq) < 0.6)).to(torch.uint8)
            self.mask[int(g.integers(hq))] = 1
        if steer:
            self.alpha = torch.from_numpy(np.where(np.arange(hq) % 2 == 0, 0.5, 0.0)).float()
            self.steer = torch.from_numpy(g.normal(size=(hq, d))).float()

    def kw(self):
        dev = lambda x: None if x is None else x.cuda()
        return dict(q=self.q.cuda(), pages=self.pages, block_table=_i32(self.table), seq_lens=_i32(self.lens), spans=dev(self.spans), head_mask=self.mask,
                    alpha=self.alpha, steer_vec=dev(self.steer), scale=self.scale)

    def check(self, out, mass, rows=None):
        out = out.double().cpu().numpy()
        probed = [] if self.mask is None else [h for h in range(self.hq) if self.mask[h]]
        assert (mass is None) == (not probed)
        scale = self.scale if self.scale > 0 else self.d ** -0.5
        loaded = q4.load(self.slabs, self.d, self.group)
        for s in range(len(self.lens)) if rows is None else rows:
            L = self.lens[s]
            if L <= 0:
                assert not out[s].any() and (mass is None or not mass[s].any())
                continue
            held = [[x[self.table[s, :-(-L // 16)]] for x in part] for part in loaded]        # [pages, Hkv, 16, D]
            for h in range(self.hq):
                kv = h // (self.hq // self.hkv)
                k, v = ([x[:, kv].reshape(-1, self.d)[:L] for x in part] for part in held)
                spans = [] if self.spans is None else self.spans[s].tolist()
                steer = 0.0 if self.alpha is None else float(self.alpha[h]) * self.steer[h].double().numpy()
                want, sums, size = q4.attend(self.q[s, h].double().numpy(), k, v, scale, steer, spans)
                most, most_mass = bounds(size, want, self.d)
                assert np.all(np.abs(out[s, h] - want) <= most), (s, h, np.abs(out[s, h] - want).max(), most.max())
                if h in probed:
                    got = mass[s, probed.index(h)].double().cpu().numpy()
                    assert np.all(np.abs(got - sums) <= most_mass), (s, h, got, sums, most_mass)


def _run(eng, case, **kw):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, mass = eng.hook_attn_decode_q4(**{**case.kw(), "status": status, **kw})
    torch.cuda.synchronize()
    return out, mass, int(status.item())


@pytest.mark.gpu
@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 1), (8, 4), (24, 3), (15, 5)])
@pytest.mark.parametrize("spans", [0, 2, 5])
def test_parity(eng, d, group, hq, hkv, spans):
    """Lengths around a page's borders, shuffled pages, NaN wherever no sequence has a token."""
    c = Case([1, 15, 16, 17, 33, 700, 100], hq, hkv, d, group, seed=hq + spans, spans=spans, steer=spans == 2)
    out, mass, status = _run(eng, c)
    assert status == 0
    c.check(out, mass)


@pytest.mark.gpu
@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("lens", [[1, 15, 16, 17, 33, 700, 100], [4000, 5, 9001, 2000], [20, 0, 300, -1]])
@pytest.mark.parametrize("spans", [0, 2, 7])
def test_parity_of_shared_pages(eng, d, group, lens, spans):
    """Tables wide enough for very long sequences: few units, whose pages are dealt out evenly, from less than one page a warp to runs that go on
    in the next unit."""
    c = Case(lens, 10, 5, d, group, seed=spans, spans=spans, steer=spans == 2, width=4000)
    out, mass, status = _run(eng, c)
    assert status == (binding.HOOK_ATTN_ERR_INVALID_ARG if min(lens) <= 0 else 0)
    c.check(out, mass)
    again = _run(eng, c)
    assert torch.equal(again[0], out) and (mass is None or torch.equal(again[1], mass))
    if min(lens) > 0:                                       # a page out of range takes its row with it, and no other
        kw = c.kw()
        kw["block_table"][2, 0] = len(c.slabs)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        bad, bad_mass = eng.hook_attn_decode_q4(**kw, status=status)
        assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS and not bad[2].any() and (mass is None or not bad_mass[2].any())
        rest = [r for r in range(len(lens)) if r != 2]
        assert torch.equal(bad[rest], out[rest]) and (mass is None or torch.equal(bad_mass[rest], mass[rest]))


@pytest.mark.gpu
@pytest.mark.parametrize("d,group", [(64, 32), (128, 32), (128, 128)])
@pytest.mark.parametrize("spans", [0, 3, 8])
def test_parity_of_many_units(eng, d, group, spans):
    """As many units as are cut into chunks; without and with a bound of the lengths."""
    lens = [int(x) for x in np.random.default_rng(2).integers(1, 400, 80)]
    lens[3], lens[50] = 1500, 1
    c = Case(lens, 8, 4, d, group, spans=spans, steer=True)
    out, mass, status = _run(eng, c)
    assert status == 0
    c.check(out, mass, rows=[0, 3, 17, 50, 79])
    out2, mass2, status = _run(eng, c, max_seq_len=1500)
    assert status == 0
    c.check(out2, mass2, rows=[0, 3, 17, 50, 79])


@pytest.mark.gpu
@pytest.mark.parametrize("kind,q_size,scale", [("steps", 1.0, 0.0), ("constant", 1.0, 0.0), ("large", 1e-3, 0.0), ("normal", 2.0 ** 40, 2.0 ** -43),
                                               ("normal", 2.0 ** -60, 2.0 ** 57), ("normal", 0.0, 0.0), ("normal", 8.0, 0.0)])
@pytest.mark.parametrize("group", [32, 128])
def test_parity_of_sizes(eng, kind, q_size, scale, group):
    """Steps from 2^-40 to 8 in one sequence, no steps at all, large values, large and small queries, sharp softmaxes."""
    c = Case([5, 300, 1000], 6, 2, 128, group, kind=kind, q_size=q_size, scale=scale, spans=2)
    out, mass, status = _run(eng, c)
    assert status == 0
    c.check(out, mass)


@pytest.mark.gpu
def test_layouts_and_preallocated_results(eng):
    c = Case([40, 3, 129], 8, 2, 64, 32, spans=2, layout="heads first")
    out, mass, _ = _run(eng, c)
    c.check(out, mass)
    ours = torch.zeros_like(out), torch.zeros_like(mass), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    got = eng.hook_attn_decode_q4(**c.kw(), out=ours[0], span_mass=ours[1], workspace=ours[2])
    assert got[0].data_ptr() == ours[0].data_ptr() and torch.equal(ours[0], out) and torch.equal(ours[1], mass)
    with pytest.raises(binding.HookAttnError) as e:
        eng.hook_attn_decode_q4(**c.kw(), workspace=ours[2][:256])
    assert e.value.code == binding.HOOK_ATTN_ERR_WORKSPACE
    with pytest.raises(binding.HookAttnError) as e:
        eng.hook_attn_decode_q4(**c.kw(), workspace=ours[2][16:])
    assert e.value.code == binding.HOOK_ATTN_ERR_WORKSPACE
    none = torch.zeros(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    out, mass = eng.hook_attn_decode_q4(q=none, pages=c.pages, block_table=torch.zeros(0, 4, dtype=torch.int32, device="cuda"),
                                        seq_lens=torch.zeros(0, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 8, 64) and mass is None


@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [6, 200])
def test_faults_become_zeros(eng, seqs):
    """Lengths that are not positive or beyond the table, pages outside the pool: status, zeros in those rows, the others as they are."""
    lens = [40 + s % 30 for s in range(seqs)]
    lens[1], lens[2] = 0, -3
    c = Case(lens, 4, 2, 128, 64, spans=2, steer=True)
    out, mass, status = _run(eng, c)
    assert status == binding.HOOK_ATTN_ERR_INVALID_ARG
    rows = [0, 1, 2, 3, 4, 5, seqs - 1]
    c.check(out, mass, rows=rows)
    kw = c.kw()
    kw["block_table"][3, 1], kw["block_table"][4, 0] = len(c.slabs), -1
    kw["seq_lens"][5] = c.table.shape[1] * 16 + 1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bad, bad_mass = eng.hook_attn_decode_q4(**kw, status=status)
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS
    for r in (3, 4, 5):
        assert not bad[r].any() and not bad_mass[r].any()
    rest = [r for r in range(seqs) if r not in (3, 4, 5)]
    assert torch.equal(bad[rest], out[rest]) and torch.equal(bad_mass[rest], mass[rest])


@pytest.mark.gpu
def test_values_that_are_not_finite_come_through(eng):
    """A NaN in a sequence's keys or values is not hidden, and stays with its KV head."""
    c = Case([64, 64, 64], 4, 2, 128, 128)
    pages = c.pages.clone()
    nan = torch.tensor([0xC0, 0x7F], dtype=torch.uint8, device="cuda")
    pages[int(c.table[0, 1]), 0, 16 * 128:16 * 128 + 2] = nan                         # step of K
    pages[int(c.table[1, 2]), 1, 16 * 128 + 64:16 * 128 + 66] = nan                   # step of V
    out, _, status = _run(eng, c, pages=pages)
    assert status == 0 and torch.isnan(out[0, :2]).all() and torch.isnan(out[1, 2:]).all()
    rest = torch.ones(3, 4, dtype=torch.bool)
    rest[0, :2] = rest[1, 2:] = False
    assert not torch.isnan(out[rest.cuda()]).any()


@pytest.mark.gpu
def test_pages_behind_four_gigabytes(eng):
    """Slabs whose offsets need more than 32 bits."""
    d, group, hkv = 128, 32, 8
    pool = (5 << 30) // (hkv * 2560)
    c = Case([100, 33], 16, hkv, d, group, spans=2)
    pages = torch.empty(pool, hkv, 2560, dtype=torch.uint8, device="cuda")
    far = {int(p): pool - 1 - i for i, p in enumerate(sorted(set(c.table[c.table >= 0].tolist())))}
    for near, to in far.items():
        pages[to] = c.pages[near]
    table = np.vectorize(lambda p: far.get(p, -1))(c.table)
    out, mass, status = _run(eng, c, pages=pages, block_table=_i32(table))
    assert status == 0
    c.check(out, mass)


@pytest.mark.gpu
def test_graphs_streams_and_repetition(eng):
    """The same bits in every run, on another stream, and from two graphs with workspaces of their own that are replayed in turn."""
    cases = [Case([300, 20, 1], 8, 2, 128, 32, spans=4, seed=3), Case([200] * 90, 8, 4, 64, 64, spans=2, seed=4)]
    want = [_run(eng, c)[:2] for c in cases]
    side = torch.cuda.Stream()
    graphs = []
    for c, (out, mass) in zip(cases, want):
        again = _run(eng, c)
        assert torch.equal(again[0], out) and torch.equal(again[1], mass)
        kw = c.kw()
        torch.cuda.synchronize()
        got = eng.hook_attn_decode_q4(**kw, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], mass)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = eng.hook_attn_decode_q4(**kw)
        graphs.append((graph, captured, kw))
    for _ in range(3):
        for graph, captured, _ in graphs:
            captured[0].fill_(7)
            graph.replay()
        torch.cuda.synchronize()
        for (_, captured, _), (out, mass) in zip(graphs, want):
            assert torch.equal(captured[0], out) and torch.equal(captured[1], mass)


@pytest.mark.gpu
def test_refused_tensors(eng):
    c = Case([20], 4, 2, 64, 32, spans=2, steer=True)
    kw = c.kw()
    for name, bad in (("q", kw["q"].float()), ("q", kw["q"].cpu()), ("pages", kw["pages"][..., :-16]), ("block_table", kw["block_table"].long()),
                      ("seq_lens", kw["seq_lens"].repeat(2)), ("spans", kw["spans"].long()), ("head_mask", kw["head_mask"].cuda()),
                      ("alpha", kw["alpha"][:2]), ("steer_vec", kw["steer_vec"].half()), ("out", kw["q"].float()), ("span_mass", kw["steer_vec"])):
        with pytest.raises(AssertionError):
            eng.hook_attn_decode_q4(**{**kw, name: bad})
