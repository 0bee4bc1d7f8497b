"""Rotary positions with several axes, appended to the paged cache: oracle pins, refusals (CPU) and GPU parity."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import ops
from paper_2603_06588_b200 import binding

from ._ops import FAKE_HANDLE, no_device, struct_fields

BF16_HALF_STEP = torch.finfo(torch.bfloat16).eps / 2
# Relative to |a| + |b| of the pair: the reduced angle is rounded to 32 bits (2 pi 2^-26), sine and cosine are off by 2 units
# (2^-22), the factor, the two products and their sum are rounded (4 x 2^-24): below 2^-21 together.
ARITHMETIC = 2.0 ** -21


# --------------------------------------------------------------------------------------------------- CPU
def test_struct_mirror():
    assert struct_fields("hook_rope_params") == [f[0] for f in binding.HookRopeParams._fields_]


def test_axes_of_pairs():
    assert ops.axis_of_pair([2, 1, 3], False) == [0, 0, 1, 2, 2, 2]
    assert ops.axis_of_pair([2, 1, 3], True) == [0, 1, 2, 0, 2, 2]
    assert ops.axis_of_pair([0, 2], True) == [1, 1]
    assert ops.axis_of_pair([5], True) == [0] * 5


def test_rotation_oracle_closed_forms():
    x = np.zeros((1, 1, 4))
    x[0, 0] = [1.0, 2.0, 3.0, 4.0]
    quarter = [math.pi / 2, 0.0]
    out, _ = ops.rotate(x, [[1]], quarter, [2], False, False, 1.0)            # pair 0 = elements 0, 2 turns by 90 degrees
    assert np.allclose(out[0, 0], [-3.0, 2.0, 1.0, 4.0])
    out, _ = ops.rotate(x, [[1]], quarter, [2], False, True, 2.0)             # pair 0 = elements 0, 1
    assert np.allclose(out[0, 0], [-4.0, 2.0, 6.0, 8.0])
    # scores depend on the difference of the positions alone
    g = np.random.default_rng(0)
    q, k, f = g.normal(size=(1, 1, 8)), g.normal(size=(1, 1, 8)), [1.0, 0.3, 0.1, 0.01]
    dot = lambda m, n: float((ops.rotate(q, [[m]], f, [4], False, False, 1.0)[0] * ops.rotate(k, [[n]], f, [4], False, False, 1.0)[0]).sum())
    assert abs(dot(7, 3) - dot(1004, 1000)) < 1e-9


def _params(**over):
    p = binding.HookRopeParams()
    p.num_seqs, p.total_q, p.num_q_heads, p.num_kv_heads, p.head_dim, p.page_size = 2, 2, 32, 8, 128, 16
    p.num_blocks, p.max_blocks_per_seq, p.rotary_dim, p.num_axes, p.factor = 64, 8, 128, 3, 1.0
    p.axis_pairs[:3] = (16, 24, 24)
    p.q = p.k = p.v = p.q_out = p.k_cache = p.v_cache = p.block_table = p.seq_lens = p.inv_freq = 0x10000
    p.q_out = 0x20000
    p.q_row_stride, p.q_head_stride, p.k_row_stride, p.k_head_stride, p.v_row_stride, p.v_head_stride = 4096, 128, 1024, 128, 1024, 128
    p.kv_block_stride, p.kv_token_stride, p.kv_head_stride = 16 * 8 * 128, 8 * 128, 128
    for k, v in over.items():
        if k == "axis_pairs":
            p.axis_pairs[:len(v)] = v
        else:
            setattr(p, k, v)
    return p


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), binding.HOOK_ATTN_ERR_CUDA),                       # valid: only the device is missing
    (dict(rotary_dim=0, num_axes=1, axis_pairs=(0,), inv_freq=None), binding.HOOK_ATTN_ERR_CUDA),
    (dict(q_out=0x10000), binding.HOOK_ATTN_ERR_CUDA),          # in place
    (dict(num_seqs=0), binding.HOOK_ATTN_ERR_INVALID_ARG),      # decode needs one row per sequence
    (dict(rotary_dim=127), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(rotary_dim=130), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(axis_pairs=(16, 24, 23)), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(axis_pairs=(-1, 41, 24)), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(axis_pairs=(2 ** 31 - 1, 2 ** 31 - 1, 66)), binding.HOOK_ATTN_ERR_INVALID_ARG),   # a sum that wraps around
    (dict(num_axes=0), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(num_axes=5), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(axis_order=2), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(pairing=-1), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(dtype=3), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(factor=float("nan")), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(inv_freq=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(q=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(num_q_heads=30), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(total_q=3), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(q_out=0x10000, dtype=binding.HOOK_DTYPE_F16), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(q_out=0x10000, q_row_stride=6144), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(kv_head_stride=0), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(head_dim=96, rotary_dim=96, axis_pairs=(16, 16, 16)), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(page_size=32), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(num_q_heads=128), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(kv_token_stride=1028), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(k_cache=0x10008), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(v=0x10001), binding.HOOK_ATTN_ERR_UNSUPPORTED),
])
def test_refusals(over, code):
    lib = binding.load_library()
    assert lib.hook_rope_append(FAKE_HANDLE, ctypes.byref(_params(**over)), None) == code


def test_no_handle_and_no_params():
    lib = binding.load_library()
    assert lib.hook_rope_append(None, ctypes.byref(_params()), None) == binding.HOOK_ATTN_ERR_INVALID_ARG
    assert lib.hook_rope_append(None, None, None) == binding.HOOK_ATTN_ERR_INVALID_ARG


# --------------------------------------------------------------------------------------------------- GPU
@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _case(q_lens, ctx, hq, hkv, d, pairs, dtype, seed=1, layout="contiguous", decode=False, fused=True, offset=0):
    g = np.random.default_rng(seed)
    rows, seqs = int(sum(q_lens)), len(q_lens)
    lens = [c + n for c, n in zip(ctx, q_lens)]
    pages = [-(-L // 16) for L in lens]
    pool = sum(pages) + 3
    order = g.permutation(pool).tolist()
    width = max(pages + [1]) + 1
    table = np.full((seqs, width), -1, dtype=np.int32)
    for s, n in enumerate(pages):
        table[s, :n], order = order[:n], order[n:]
    t = lambda *shape: torch.from_numpy(g.normal(size=shape)).to(dtype)
    if fused:                                                   # slices of one projection, `offset` elements into their rows
        qkv = t(rows, offset + (hq + 2 * hkv) * d)[:, offset:].unflatten(1, (hq + 2 * hkv, d))
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        q, k, v = t(rows, hq, d), t(rows, hkv, d), t(rows, hkv, d)
    shape = {"contiguous": (pool, 2, 16, hkv, d), "heads first": (pool, 2, hkv, 16, d), "padded": (pool, 2, 16, hkv, d + 8)}[layout]
    cache = torch.full(shape, 7.0, dtype=torch.bfloat16)
    return dict(q=q, k=k, v=v, cache=cache, block_table=torch.from_numpy(table), seq_lens=torch.tensor(lens, dtype=torch.int32),
                cu_q_lens=None if decode else torch.tensor([0] + list(np.cumsum(q_lens)), dtype=torch.int32), layout=layout, d=d)


def _views(cache, layout, d):
    k, v = cache[:, 0], cache[:, 1]
    if layout == "heads first":
        return k.transpose(1, 2), v.transpose(1, 2)
    return k[..., :d], v[..., :d]


def _check(eng, c, inv_freq, axis_pairs, cyclic=False, adjacent=False, factor=1.0, positions=None, in_place=False, expect_status=0):
    dev = lambda x: None if x is None else x.cuda()
    fused = c["q"].untyped_storage().data_ptr() == c["k"].untyped_storage().data_ptr() and c["q"].numel()
    if fused:                                                   # keep the strides on the device
        base = torch.as_strided(c["q"], (c["q"].untyped_storage().nbytes() // c["q"].element_size(),), (1,), 0).cuda()
        q, k, v = (torch.as_strided(base, x.shape, x.stride(), x.storage_offset()) for x in (c["q"], c["k"], c["v"]))
    else:
        q, k, v = c["q"].cuda(), c["k"].cuda(), c["v"].cuda()
    rows, hq, d = q.shape
    cache = c["cache"].cuda()
    kc, vc = _views(cache, c["layout"], d)
    q_out = q if in_place else torch.full((rows, hq, d), 5.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = eng.hook_rope_append(
        q=q, k=k, v=v, k_cache=kc, v_cache=vc, block_table=c["block_table"].cuda(), seq_lens=c["seq_lens"].cuda(), cu_q_lens=dev(c["cu_q_lens"]),
        positions=dev(positions), inv_freq=torch.tensor(inv_freq, dtype=torch.float32, device="cuda"), axis_pairs=axis_pairs,
        axis_order=binding.HOOK_ROPE_AXES_CYCLIC if cyclic else binding.HOOK_ROPE_AXES_BLOCKED,
        pairing=binding.HOOK_ROPE_PAIR_ADJACENT if adjacent else binding.HOOK_ROPE_PAIR_HALVES, factor=factor, q_out=q_out, status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == expect_status
    freq = np.asarray(inv_freq, dtype=np.float32).astype(np.float64)
    lens, table = c["seq_lens"].tolist(), c["block_table"].tolist()
    cu = list(range(len(lens) + 1)) if c["cu_q_lens"] is None else c["cu_q_lens"].tolist()
    places = ops.row_places(lens, cu, table, len(cache))
    pos = positions.tolist() if positions is not None else [[0 if p is None else p[0] for p in places] + [0] * (rows - len(places))] * len(axis_pairs)
    fac = float(np.float32(factor))
    want_q, scale_q = ops.rotate(c["q"].double().numpy(), pos, freq, axis_pairs, cyclic, adjacent, fac)
    want_k, scale_k = ops.rotate(c["k"].double().numpy(), pos, freq, axis_pairs, cyclic, adjacent, fac)
    got_q = got.double().cpu().numpy()
    want_cache = c["cache"].clone()
    wk, wv = _views(want_cache, c["layout"], d)
    gk, gv = _views(cache.cpu(), c["layout"], d)
    for t in range(rows):
        if t >= len(places):                                    # behind the last sequence
            assert (got_q[t] == 5.0).all()
            continue
        if places[t] is None:
            assert (got_q[t] == 0.0).all()
            continue
        _, page, slot = places[t]
        assert np.all(np.abs(got_q[t] - want_q[t]) <= np.abs(want_q[t]) * BF16_HALF_STEP + scale_q[t] * ARITHMETIC)
        row = gk[page, slot].double().numpy()
        assert np.all(np.abs(row - want_k[t]) <= np.abs(want_k[t]) * BF16_HALF_STEP + scale_k[t] * ARITHMETIC)
        wk[page, slot] = gk[page, slot]
        wv[page, slot] = c["v"][t].to(torch.bfloat16)           # one rounding, nothing else
    assert torch.equal(cache.cpu().view(torch.int16), want_cache.view(torch.int16))      # no other element of the cache has changed


def _freq(pairs, base=10000.0):
    return [base ** (-i / max(1, pairs)) for i in range(pairs)]


def _axes_positions(rows, axes, seed, top=1 << 20):
    return torch.from_numpy(np.random.default_rng(seed).integers(0, top, (axes, rows))).int()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,rot,axis_pairs,cyclic", [
    (128, 128, (64,), False), (128, 128, (16, 24, 24), False), (128, 128, (24, 20, 20), True), (64, 64, (8, 12, 12), True),
    (64, 40, (8, 6, 6), True), (128, 32, (4, 4, 4, 4), False), (64, 16, (8,), False), (64, 6, (1, 0, 2), False), (128, 52, (9, 17), True), (128, 2, (1,), True),
    (128, 126, (40, 23), False)])
def test_ragged_prompts(eng, dtype, adjacent, d, rot, axis_pairs, cyclic):
    """Packed prompts with and without context, a sequence without rows, rows that end inside pages."""
    c = _case([5, 0, 17, 1, 40], [0, 9, 31, 16, 3], 6, 2, d, rot // 2, dtype, seed=rot)
    _check(eng, c, _freq(rot // 2), axis_pairs, cyclic, adjacent, 1.0 if len(axis_pairs) == 1 else 0.75, _axes_positions(63, len(axis_pairs), rot))


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["contiguous", "heads first", "padded"])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (14, 2), (64, 8)])
def test_decode_rows(eng, layout, hq, hkv):
    """One row per sequence at its place, on every cache layout."""
    c = _case([1] * 7, [0, 1, 15, 16, 17, 255, 1000], hq, hkv, 128, 64, torch.bfloat16, layout=layout, decode=True)
    _check(eng, c, _freq(64), (64,))


@pytest.mark.gpu
@pytest.mark.parametrize("rot", [0, 64])
@pytest.mark.parametrize("offset", [0, 1, 2, 4])
def test_unaligned_rows(eng, rot, offset):
    """q, k and v start anywhere in the rows of a wider buffer: no 16-byte alignment."""
    c = _case([9, 3], [0, 20], 4, 4, 64, rot // 2, torch.bfloat16, offset=offset)
    _check(eng, c, _freq(rot // 2), (rot // 2,))


@pytest.mark.gpu
@pytest.mark.parametrize("adjacent", [False, True])
def test_in_place_queries(eng, adjacent):
    c = _case([9, 3], [0, 20], 4, 2, 128, 64, torch.bfloat16, fused=False)
    _check(eng, c, _freq(64), (64,), adjacent=adjacent, in_place=True)
    c = _case([1], [20], 4, 2, 128, 64, torch.bfloat16, fused=False, decode=True)
    c["q"] = torch.as_strided(c["q"], (1, 4, 128), (7, 128, 1))   # the stride of a single row is of no account
    _check(eng, c, _freq(64), (64,), adjacent=adjacent, in_place=True)


@pytest.mark.gpu
def test_a_factor_of_zero_selects_one(eng):
    c = _case([3], [1], 2, 1, 64, 32, torch.bfloat16)
    kw = dict(q=c["q"].cuda(), k=c["k"].cuda(), v=c["v"].cuda(), block_table=c["block_table"].cuda(), seq_lens=c["seq_lens"].cuda(),
              cu_q_lens=c["cu_q_lens"].cuda(), inv_freq=torch.tensor(_freq(32), device="cuda"))
    got = [eng.hook_rope_append(k_cache=k, v_cache=v, factor=f, **kw) for f in (0.0, 1.0) for k, v in [_views(c["cache"].cuda(), "contiguous", 64)]]
    assert torch.equal(*got) and got[0].any()


@pytest.mark.gpu
def test_far_and_negative_positions(eng):
    c = _case([40], [0], 2, 1, 128, 64, torch.float32)
    pos = torch.from_numpy(np.random.default_rng(3).integers(-(1 << 24), 1 << 24, (3, 40))).int()
    _check(eng, c, _freq(64), (16, 24, 24), positions=pos)


@pytest.mark.gpu
def test_rows_behind_the_last_sequence_stay(eng):
    c = _case([3, 4], [5, 0], 4, 2, 64, 32, torch.bfloat16, fused=False)
    c["cu_q_lens"][2] = 5                                       # two of the seven rows are padding
    c["seq_lens"][1] = 2
    _check(eng, c, _freq(32), (32,))


@pytest.mark.gpu
@pytest.mark.parametrize("fault", ["page", "negative page", "too long", "more rows than keys", "empty"])
def test_broken_rows_are_zeroed_and_append_nothing(eng, fault):
    c = _case([3, 4, 2], [5, 12, 0], 4, 2, 64, 32, torch.bfloat16)
    if fault == "page":
        c["block_table"][1, 0] = 1 << 20
    elif fault == "negative page":
        c["block_table"][1, 0] = -1
    elif fault == "too long":
        c["seq_lens"][1] = 16 * c["block_table"].shape[1] + 1
    elif fault == "more rows than keys":
        c["seq_lens"][1] = 3
    else:
        c["seq_lens"][1] = 0
    _check(eng, c, _freq(32), (32,), expect_status=binding.HOOK_ATTN_ERR_BOUNDS)


@pytest.mark.gpu
def test_many_sequences(eng):
    """More sequences than a block has threads: the search for a row's sequence goes on."""
    n = [i % 3 for i in range(700)]
    c = _case(n, [i % 5 for i in range(700)], 1, 1, 64, 8, torch.bfloat16)
    _check(eng, c, _freq(8), (8,))


@pytest.mark.gpu
def test_tensors_elsewhere_are_refused(eng):
    c = _case([1], [3], 2, 2, 64, 32, torch.bfloat16, decode=True)
    k, v = _views(c["cache"], "contiguous", 64)
    kw = dict(q=c["q"], k=c["k"], v=c["v"], k_cache=k, v_cache=v, block_table=c["block_table"], seq_lens=c["seq_lens"], inv_freq=torch.ones(32))
    with pytest.raises(AssertionError):
        eng.hook_rope_append(**kw)
    with pytest.raises(AssertionError):
        eng.hook_rope_append(**dict({n: t.cuda() for n, t in kw.items()}, seq_lens=c["seq_lens"]))


@pytest.mark.gpu
def test_nothing_to_do(eng):
    c = _case([0, 0], [3, 4], 2, 2, 64, 32, torch.bfloat16)
    _check(eng, c, _freq(32), (32,))


@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [31, 128, 129, 1025, 4100])
def test_sequences_narrowed_down(eng, seqs):
    """More of them than a warp looks at side by side, many without a row, in runs too."""
    g = np.random.default_rng(seqs)
    q_lens = g.integers(0, 4, seqs) * (g.random(seqs) < 0.6)
    q_lens[seqs // 3:seqs // 2] = 0
    q_lens[-1] = g.integers(0, 2)
    _check(eng, _case(q_lens.tolist(), g.integers(0, 40, seqs).tolist(), 2, 1, 64, 32, torch.bfloat16), _freq(32), (32,))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
def test_the_farthest_positions(eng, dtype, adjacent):
    """Positions next to the last integers.  The product with the frequency, the one with 1 / (2 pi) and that constant are rounded to 53 bits
    before the whole turns go: 3 x 2^-53 x 2^31 f = 3 f 2^-22 rad, for f <= 1/16 below 0.19 x 2^-22.  Beside it the reduced angle (2 pi 2^-26 =
    0.4 x 2^-22), sine and cosine (a unit: 2^-24), the factor, a product and the sum (3 x 2^-24): 1.6 x 2^-22 together, below 2^-21."""
    c = _case([40], [0], 2, 1, 64, 32, dtype)
    g = np.random.default_rng(3)
    pos = np.stack([2 ** 31 - 1 - g.integers(0, 100, 40), -2 ** 31 + g.integers(0, 100, 40), g.integers(-2 ** 31, 2 ** 31, 40)])
    _check(eng, c, [f / 16 for f in _freq(32, 4.0)], (8, 12, 12), adjacent=adjacent, positions=torch.from_numpy(pos).int())


def test_oracle_of_far_positions():
    """Against angles reduced in whole numbers: 2 pi to 60 digits."""
    tau = 6283185307179586476925286766559005768394338798750211641949889
    x = np.array([[[1.0, 0.0]]])
    for pos, freq in ((2 ** 31 - 1, 1 - 2.0 ** -24), (-2 ** 31, 0.75), (2 ** 31 - 12345, 2.0 ** -7 + 2.0 ** -30)):
        angle = pos * int(freq * 2 ** 60) * 10 ** 60 % (tau * 2 ** 60) / (10 ** 60 * 2 ** 60)
        out, _ = ops.rotate(x, [[pos]], [freq], [1], False, False, 1.0)
        assert np.abs(out[0, 0] - [math.cos(angle), math.sin(angle)]).max() < 2.0 ** -50


def _long_case(rows, pairs, dtype, seed, broken=True, **kw):
    """Packed prompts of some ten rows each, two of them broken, five rows of padding at the end."""
    g = np.random.default_rng(seed)
    n = g.integers(0, 21, rows // 8)
    n = n[:int(np.searchsorted(np.cumsum(n), rows - 50))].tolist()
    n.append(rows - sum(n))
    c = _case(n, g.integers(0, 40, len(n)).tolist(), 2, 1, 64, pairs, dtype, seed=seed, **kw)
    if broken:
        c["block_table"][len(n) // 3, 0] = -1
        c["seq_lens"][len(n) // 2] = 16 * c["block_table"].shape[1] + 1
        c["cu_q_lens"][-1] -= 5
        c["seq_lens"][-1] -= 5
    return c


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("axis_pairs", [(8, 12, 12), (3, 9), (5, 0, 1), (16, 15)])
def test_several_rows_to_a_block(eng, dtype, adjacent, axis_pairs):
    """Runs of eight, four, two and one elements, good and broken rows and padding side by side."""
    c = _long_case(2531, sum(axis_pairs), dtype, sum(axis_pairs))
    assert c["cu_q_lens"][-1] == 2526
    _check(eng, c, _freq(sum(axis_pairs)), axis_pairs, True, adjacent, 0.75, _axes_positions(2531, len(axis_pairs), 3), expect_status=binding.HOOK_ATTN_ERR_BOUNDS)


@pytest.mark.gpu
@pytest.mark.parametrize("axis_pairs,dtype", [((8, 12, 12), torch.bfloat16), ((5, 0, 1), torch.float32)])
def test_as_many_rows_to_a_block_as_there_can_be(eng, axis_pairs, dtype):
    c = _long_case(10007, sum(axis_pairs), dtype, 7)
    _check(eng, c, _freq(sum(axis_pairs)), axis_pairs, positions=_axes_positions(10007, len(axis_pairs), 3), expect_status=binding.HOOK_ATTN_ERR_BOUNDS)


@pytest.mark.gpu
@pytest.mark.parametrize("adjacent", [False, True])
def test_in_place_queries_of_several_rows_to_a_block(eng, adjacent):
    c = _long_case(2503, 32, torch.bfloat16, 9, broken=False, fused=False)
    _check(eng, c, _freq(32), (32,), adjacent=adjacent, in_place=True)


@pytest.mark.gpu
def test_as_many_sequences_as_there_can_be(eng):
    """65535 of them, most without a row; and a cache whose last pages lie behind the first 2^32 elements."""
    seqs, rows, pages, i32 = 65535, 3000, 2 ** 32 // (2 * 16 * 8 * 128) + 3000, dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    at = torch.randint(0, seqs, (rows,), generator=g, device="cuda").sort().values
    n = torch.bincount(at, minlength=seqs)
    cu = torch.zeros(seqs + 1, **i32)
    cu[1:] = n.cumsum(0)
    lens = (n + torch.randint(0, 30, (seqs,), generator=g, device="cuda")).int()
    table = torch.full((seqs, 3), -1, **i32)
    live = (torch.arange(3, device="cuda") * 16 < lens[:, None]) & (n > 0)[:, None]
    table[live] = (pages - 1 - torch.randperm(int(live.sum()), generator=g, device="cuda")).int()
    q, k, v = (torch.randn(rows, h, 128, generator=g, device="cuda").bfloat16() for h in (8, 8, 8))
    cache = torch.empty((pages, 2, 16, 8, 128), dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, **i32)
    freq = torch.tensor(_freq(64), device="cuda")
    got = eng.hook_rope_append(q=q, k=k, v=v, k_cache=cache[:, 0], v_cache=cache[:, 1], block_table=table, seq_lens=lens, cu_q_lens=cu, inv_freq=freq, status=status)
    pos = (lens[at] - cu[at + 1] + torch.arange(rows, device="cuda")).long()
    page = table[at, pos // 16].long()
    assert int(page.min()) * 2 * 16 * 8 * 128 > 2 ** 31 and int(page.max()) == pages - 1 and int(status.item()) == 0
    assert torch.equal(cache[page, 1, pos % 16], v)
    angle = pos[:, None].double() * freq.double()
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    for res, x in ((got, q), (cache[page, 0, pos % 16], k)):
        z = torch.complex(x[..., :64].double(), x[..., 64:].double()) * turn
        want, scale = torch.cat([z.real, z.imag], -1), x[..., :64].double().abs() + x[..., 64:].double().abs()
        assert ((res.double() - want).abs() <= want.abs() * BF16_HALF_STEP + torch.cat([scale, scale], -1) * ARITHMETIC).all()
