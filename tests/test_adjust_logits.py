"""Penalties, biases and grammar masks on logits: oracle pins, refusals (CPU) and GPU parity."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ops
from paper_2603_06588_b200 import binding

from ._ops import FAKE_HANDLE, no_device, struct_fields

# Relative to the sum of the magnitudes of a value's terms: the reciprocal, the product with it, the one with the count, the two sums and the
# addition of the bias are each rounded to 24 bits: 6 x 2^-24 < 2^-21.
ARITHMETIC = 2.0 ** -21
SMALLEST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}    # half a step of the numbers next to zero


# --------------------------------------------------------------------------------------------------- CPU
def test_struct_mirror():
    assert struct_fields("hook_logits_params") == [f[0] for f in binding.HookLogitsParams._fields_]


def test_oracle_closed_forms():
    x = np.array([[2.0, -2.0, 1.0, 0.5, 3.0]])
    out, _ = ops.adjust_logits(x, tokens=[[0, 1, 4, 4, -1, 7]], prompt_lens=[1], total_lens=[6], repetition=[2.0], presence=[0.25], frequency=[0.5],
                               bias=[[(3, 1.0), (3, 2.0), (9, 5.0)]], mask=np.array([[1, 1, 0, 1, 1]], dtype=bool))
    assert out[0].tolist() == [1.0, -4.0 - 0.75, -np.inf, 2.5, 1.5 - 1.25]
    same, _ = ops.adjust_logits(x, mask=np.zeros((1, 5), dtype=bool), mask_rows=[-1])
    assert np.array_equal(same, x)


def _params(**over):
    p = binding.HookLogitsParams()
    p.num_rows, p.vocab_size, p.max_tokens, p.num_bias, p.num_masks = 2, 1000, 64, 4, 2
    p.logits, p.out, p.logits_row_stride, p.out_row_stride = 0x10000, 0x20000, 1000, 1000
    p.tokens = p.prompt_lens = p.total_lens = p.bias_offsets = p.bias_tokens = p.bias_values = p.mask = 0x30000
    p.tokens_row_stride, p.mask_row_stride = 64, 32
    for k, v in over.items():
        setattr(p, k, v)
    return p


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), binding.HOOK_ATTN_ERR_CUDA),
    (dict(out=0x10000), binding.HOOK_ATTN_ERR_CUDA),
    (dict(tokens=None, prompt_lens=None, total_lens=None), binding.HOOK_ATTN_ERR_CUDA),
    (dict(num_rows=-1), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(vocab_size=0), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(dtype=7), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(logits=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(out_row_stride=999), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(prompt_lens=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(tokens_row_stride=-1), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(tokens_row_stride=0, mask_row_stride=0), binding.HOOK_ATTN_ERR_CUDA),
    (dict(bias_values=None), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(mask_row_stride=-1), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(num_masks=1), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(out=0x10000, out_dtype=binding.HOOK_DTYPE_F32), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(out=0x10000, out_row_stride=1008), binding.HOOK_ATTN_ERR_INVALID_ARG),
    (dict(out_dtype=binding.HOOK_DTYPE_F16), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(vocab_size=(1 << 20) + 1, logits_row_stride=1 << 21, out_row_stride=1 << 21, mask_row_stride=1 << 16), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(max_tokens=1 << 20, tokens_row_stride=1 << 20), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(num_rows=65536), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(logits=0x10001), binding.HOOK_ATTN_ERR_UNSUPPORTED),
    (dict(out=0x20002, dtype=binding.HOOK_DTYPE_F32, out_dtype=binding.HOOK_DTYPE_F32), binding.HOOK_ATTN_ERR_UNSUPPORTED),
])
def test_refusals(over, code):
    assert binding.load_library().hook_adjust_logits(FAKE_HANDLE, ctypes.byref(_params(**over)), None) == code


# --------------------------------------------------------------------------------------------------- GPU
@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _bits(mask):
    """Boolean ``[masks, vocab]`` as int32 words, lowest bit first."""
    words = -(-mask.shape[1] // 32)
    padded = np.zeros((mask.shape[0], words * 32), dtype=np.uint8)
    padded[:, :mask.shape[1]] = mask
    return torch.from_numpy(np.packbits(padded, axis=1, bitorder="little").view(np.int32).copy())


def _check(eng, x, out_dtype=None, tokens=None, prompt=None, total=None, rep=None, pres=None, freq=None, bias=None, mask=None, mask_rows=None,
           in_place=False, pad=0, out_pad=0, expect_status=0, untouched=()):
    rows, vocab = x.shape
    out_dtype = out_dtype or x.dtype
    i32 = lambda a: None if a is None else torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    f32 = lambda a: None if a is None else torch.tensor(a, dtype=torch.float32, device="cuda")
    wide = torch.full((rows, vocab + pad), 3.0, dtype=x.dtype, device="cuda")
    wide[:, :vocab] = x.cuda()
    logits = wide[:, :vocab]
    out_wide = wide if in_place else torch.full((rows, vocab + out_pad), 3.0, dtype=out_dtype, device="cuda")
    out = out_wide[:, :vocab]
    kw = {}
    if bias is not None:
        kw = dict(bias_offsets=i32(np.cumsum([0] + [len(b) for b in bias])), bias_tokens=i32([t for b in bias for t, _ in b] or np.zeros(0)),
                  bias_values=f32([v for b in bias for _, v in b]))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = eng.hook_adjust_logits(logits, out=None if in_place else out, tokens=i32(tokens), prompt_lens=i32(prompt), total_lens=i32(total),
                                 repetition=f32(rep), presence=f32(pres), frequency=f32(freq), mask=None if mask is None else _bits(mask).cuda(),
                                 mask_rows=i32(mask_rows), status=status, **kw)
    torch.cuda.synchronize()
    assert int(status.item()) == expect_status and got.data_ptr() == out.data_ptr()
    r32 = lambda a: None if a is None else np.asarray(a, dtype=np.float32).astype(np.float64)
    live = [r for r in range(rows) if r not in untouched]
    pick = lambda a: None if a is None else [a[r] for r in live]
    bias32 = None if bias is None else [[(t, float(np.float32(v))) for t, v in bias[r]] for r in live]
    if mask is not None and mask_rows is None:
        mask_rows = list(range(rows))
    want, scale = ops.adjust_logits(x.double().numpy()[live], tokens=pick(tokens), prompt_lens=pick(prompt), total_lens=pick(total),
                                    repetition=pick(r32(rep)), presence=pick(r32(pres)), frequency=pick(r32(freq)), bias=bias32, mask=mask,
                                    mask_rows=pick(mask_rows))
    top = torch.finfo(out_dtype)
    want[np.abs(want) >= top.max * (1 + top.eps / 4)] *= np.inf          # rounded to out's type, these are infinite
    res = out.double().cpu().numpy()
    for r in untouched:
        assert np.array_equal(res[r], np.full(vocab, 3.0) if not in_place else x[r].double().numpy())
    res = res[live]
    fine = np.isfinite(want)
    assert np.array_equal(res[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]) and np.array_equal(np.isnan(res), np.isnan(want))
    tol = np.abs(want) * (torch.finfo(out_dtype).eps / 2) + scale * ARITHMETIC + SMALLEST[out_dtype]
    assert np.all(np.abs(res[fine] - want[fine]) <= tol[fine])
    if out_wide.shape[1] > vocab:
        assert (out_wide[:, vocab:] == 3.0).all()
    return got


def _random(rows, vocab, dtype, hist, seed, bias=0):
    g = np.random.default_rng(seed)
    x = torch.from_numpy(g.normal(size=(rows, vocab)) * 3).to(dtype)
    tokens = (g.random((rows, max(1, hist))) ** 3 * vocab).astype(np.int64)
    total = g.integers(0, hist + 1, rows)
    prompt = (total * g.random(rows)).astype(np.int64)
    b = [[(int(t), float(v)) for t, v in zip(g.integers(0, vocab, g.integers(0, bias + 1)), g.normal(size=bias) * 4)] for _ in range(rows)] if bias else None
    return g, x, dict(tokens=tokens, prompt=prompt, total=total, rep=1 + g.random(rows), pres=g.random(rows), freq=g.random(rows), bias=b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, None), (torch.bfloat16, torch.float32), (torch.float16, None), (torch.float16, torch.float32),
                                       (torch.float32, None)])
@pytest.mark.parametrize("vocab", [1, 31, 33, 1000, 8192, 20011])
def test_everything_on(eng, dtype, out, vocab):
    """Odd vocabularies make every row start at another alignment; history with repeats; biases with tokens named twice."""
    g, x, kw = _random(5, vocab, dtype, 300, vocab, bias=40)
    mask = g.random((3, vocab)) < 0.7
    _check(eng, x, out, mask=mask, mask_rows=[2, -1, 0, 2, 1], **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, None), (torch.bfloat16, torch.float32), (torch.float16, torch.float32), (torch.float32, None)])
@pytest.mark.parametrize("vocab", [1, 33, 777, 20011, 300007])
def test_everything_on_with_long_histories(eng, dtype, out, vocab):
    """Rows whose history is shared out; rows without one, and one that breaks off inside a load, beside them."""
    g, x, kw = _random(4, vocab, dtype, 6007, vocab + 1, bias=70)
    kw["total"][:3] = 6007, 0, 4999
    kw["prompt"][:3] = 100, 0, 4998
    _check(eng, x, out, mask=g.random((3, vocab)) < 0.7, mask_rows=[2, -1, 0, 1], **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("hist", [1, 255, 4097, 50000])
def test_long_histories(eng, hist):
    _, x, kw = _random(3, 50021, torch.bfloat16, hist, hist)
    kw["total"][0], kw["prompt"][0] = hist, 0
    _check(eng, x, torch.float32, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 2, 150, 600, 900])
def test_many_rows(eng, rows):
    g, x, kw = _random(rows, 3001, torch.float32, 64, rows, bias=3)
    _check(eng, x, mask=g.random((rows, 3001)) < 0.5, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out,pad,out_pad,in_place", [
    (torch.bfloat16, torch.float32, 0, 0, False), (torch.bfloat16, None, 0, 0, True), (torch.float16, None, 5, 3, False),
    (torch.float16, torch.float32, 0, 0, False), (torch.float32, None, 0, 0, False), (torch.float32, None, 7, 7, True), (torch.float32, None, 1, 2, False)])
@pytest.mark.parametrize("rows,vocab,hist", [(100, 50023, 300), (130, 20005, 1500), (37, 131072, 9001), (300, 20000, 8193), (9700, 301, 20)])
def test_large_batches(eng, dtype, out, pad, out_pad, in_place, rows, vocab, hist):
    """Long stretches of both lengths and short ones, rows without a history, refused and unaligned rows."""
    g, x, kw = _random(rows, vocab, dtype, hist, rows + vocab, bias=20)
    kw["total"][:4] = hist, 0, 1, hist - 1
    kw["prompt"][:4] = hist // 2, 0, 0, hist - 1
    kw["total"][rows // 2] = hist + 1
    kw["tokens"][4, ::3] = vocab + 5                            # placeholders
    _check(eng, x, out, mask=g.random((5, vocab)) < 0.6, mask_rows=g.integers(-1, 5, rows).tolist(), pad=pad, out_pad=out_pad, in_place=in_place,
           untouched=(rows // 2,), expect_status=binding.HOOK_ATTN_ERR_BOUNDS, **kw)


@pytest.mark.gpu
def test_large_batch_with_many_different_tokens(eng):
    """A row whose stretches have more words than a warp lists, beside rows that repeat one token."""
    rows, vocab, hist = 120, 40960, 20000
    g, x, kw = _random(rows, vocab, torch.bfloat16, hist, 3)
    kw["total"][:3] = hist
    kw["prompt"][:3] = 0, hist, hist // 2
    kw["tokens"][0] = g.permutation(vocab)[:hist]
    kw["tokens"][1], kw["tokens"][2] = 77, np.arange(hist) // 7
    _check(eng, x, torch.float32, **kw)


@pytest.mark.gpu
def test_large_vocabulary(eng):
    g, x, kw = _random(2, (1 << 20) - 3, torch.bfloat16, 2000, 5, bias=500)
    _check(eng, x, torch.float32, mask=g.random((2, x.shape[1])) < 0.5, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("pad,out_pad", [(0, 0), (24, 0), (5, 3), (1, 0), (0, 8)])
@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.float32), (torch.float32, None), (torch.float16, None)])
@pytest.mark.parametrize("hist", [100, 5000])
def test_strided_rows(eng, pad, out_pad, dtype, out, hist):
    g, x, kw = _random(4, 1021, dtype, hist, 11, bias=5)
    _check(eng, x, out, mask=g.random((4, 1021)) < 0.5, pad=pad, out_pad=out_pad, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_in_place(eng, dtype):
    g, x, kw = _random(4, 9001, dtype, 100, 12, bias=5)
    _check(eng, x, mask=g.random((4, 9001)) < 0.5, in_place=True, pad=7, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("only", ["rep", "pres", "freq", "bias", "mask", "nothing", "tokens"])
def test_one_edit_at_a_time(eng, only):
    g, x, kw = _random(3, 777, torch.float32, 100, 13, bias=9)
    history = {k: kw[k] for k in ("tokens", "prompt", "total")}
    args = {"bias": dict(bias=kw["bias"]), "mask": dict(mask=g.random((3, 777)) < 0.5), "nothing": {}, "tokens": history}
    _check(eng, x, **args.get(only) or dict(history, **({only: kw[only]} if only in kw else {})))


@pytest.mark.gpu
def test_masks_that_leave_nothing_infinities_and_nan(eng):
    x = torch.zeros(3, 40)
    x[0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), torch.finfo(torch.float32).min])
    x[1] = x[0]
    x[2] = float("nan")
    mask = np.ones((2, 40), dtype=bool)
    mask[1] = False
    tokens = [[0, 1, 3, 3]] * 3
    _check(eng, x, tokens=tokens, prompt=[1] * 3, total=[4] * 3, freq=[0.5] * 3, rep=[1.25] * 3, mask=mask, mask_rows=[0, 1, 1])


@pytest.mark.gpu
def test_tokens_and_biases_outside_the_vocabulary(eng):
    x = torch.randn(2, 50, generator=torch.Generator().manual_seed(1))
    tokens = [[-1, 50, 2 ** 31 - 1, -2 ** 31, 7], [50, 51, 52, 53, 54]]
    _check(eng, x, tokens=tokens, prompt=[0, 2], total=[5, 5], freq=[0.5, 0.5], rep=[2.0, 2.0])
    _check(eng, x, bias=[[(3, 1.0), (-1, 9.0)], [(50, 2.0), (49, 1.0)]], expect_status=binding.HOOK_ATTN_ERR_BOUNDS)


@pytest.mark.gpu
@pytest.mark.parametrize("entries", [2047, 2048])
def test_longest_list_of_biases(eng, entries):
    x = torch.randn(2, 3001, generator=torch.Generator().manual_seed(1))
    g = np.random.default_rng(entries)
    bias = [[(5, 1.0)], [(int(t), float(v)) for t, v in zip(g.integers(0, 3001, entries), g.normal(size=entries))]]
    _check(eng, x, tokens=[[5, 5]] * 2, prompt=[0, 0], total=[2, 2], freq=[1.0, 1.0], bias=bias,
           **(dict(expect_status=binding.HOOK_ATTN_ERR_BOUNDS, untouched=(1,)) if entries > 2047 else {}))


@pytest.mark.gpu
@pytest.mark.parametrize("over", [dict(total=[5, 9]), dict(total=[5, -1]), dict(prompt=[0, 6]), dict(prompt=[0, -1]), dict(mask_rows=[0, 2])])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("width", [8, 5000])
def test_broken_rows_are_left_alone(eng, over, in_place, width):
    x = torch.randn(2, 50, generator=torch.Generator().manual_seed(1))
    over = {k: [width + 1 if v == 9 else v for v in o] for k, o in over.items()}
    kw = dict(tokens=[[1, 2, 3, 4, 5, 6, 7, 8] + [0] * (width - 8)] * 2, prompt=[0, 0], total=[5, 5], freq=[0.5, 0.5], mask=np.arange(100).reshape(2, 50) % 3 > 0, mask_rows=[1, 0])
    _check(eng, x, expect_status=binding.HOOK_ATTN_ERR_BOUNDS, untouched=(1,), in_place=in_place, **dict(kw, **over))


@pytest.mark.gpu
def test_shared_histories_and_rows_that_overlap(eng):
    """Rows may share one history and one mask by a stride of 0; logits that overlap are refused."""
    x = torch.randn(3, 100, generator=torch.Generator().manual_seed(4)).cuda()
    tokens, lens = torch.arange(20, dtype=torch.int32, device="cuda").expand(3, 20), torch.full((3,), 20, dtype=torch.int32, device="cuda")
    freq, mask = torch.full((3,), 0.5, device="cuda"), torch.full((1, 4), 0x7fff00ff, dtype=torch.int32, device="cuda")
    got = eng.hook_adjust_logits(x, out=torch.empty_like(x), tokens=tokens, prompt_lens=lens - 10, total_lens=lens, frequency=freq, mask=mask.expand(3, 4))
    want = x.clone()
    want[:, 10:20] -= 0.5
    bits = torch.arange(100, device="cuda")
    want[:, (0x7fff00ff >> (bits % 32)) & 1 == 0] = float("-inf")
    assert torch.equal(got, want)
    with pytest.raises(AssertionError):
        eng.hook_adjust_logits(x[:1].expand(3, 100), out=torch.empty_like(x))
    with pytest.raises(AssertionError):
        eng.hook_adjust_logits(x.cpu())
    with pytest.raises(AssertionError):
        eng.hook_adjust_logits(x, tokens=tokens.cpu(), prompt_lens=lens, total_lens=lens)


@pytest.mark.gpu
def test_same_bits_every_time(eng):
    g, x, kw = _random(7, 20011, torch.bfloat16, 3000, 21, bias=60)
    first = _check(eng, x, torch.float32, **kw).clone()
    for _ in range(3):
        assert torch.equal(_check(eng, x, torch.float32, **kw), first)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out,pad,in_place", [(torch.bfloat16, torch.float32, 0, False), (torch.float16, None, 3, True), (torch.float32, None, 0, True)])
@pytest.mark.parametrize("rows,vocab,hist", [(13, 128000, 12289), (60, 32771, 20000), (130, 16384, 13000), (100, 16400, 12288)])
def test_long_histories_in_large_batches(eng, dtype, out, pad, in_place, rows, vocab, hist):
    """Stretches of 32768 values: rows of several, of one and of part of one."""
    g, x, kw = _random(rows, vocab, dtype, hist, rows + vocab, bias=20)
    kw["total"][:4] = hist, 0, 1, hist - 1
    kw["prompt"][:4] = hist // 2, 0, 0, hist - 1
    kw["total"][rows // 2] = -1
    _check(eng, x, out, mask=g.random((5, vocab)) < 0.6, mask_rows=g.integers(-1, 5, rows).tolist(), pad=pad, in_place=in_place,
           untouched=(rows // 2,), expect_status=binding.HOOK_ATTN_ERR_BOUNDS, **kw)


@pytest.mark.gpu
def test_offsets_into_an_empty_list_of_biases(eng):
    x = torch.randn(2, 50, generator=torch.Generator().manual_seed(1)).cuda()
    t = lambda a, dtype=torch.int32: torch.tensor(a, dtype=dtype, device="cuda")
    kw = dict(bias_tokens=t([]), bias_values=t([], torch.float32))
    for offsets, code in (([0, 0, 0], 0), ([0, 0, 3], binding.HOOK_ATTN_ERR_BOUNDS)):
        status, out = t([0]), torch.full_like(x, 3.0)
        eng.hook_adjust_logits(x, out=out, bias_offsets=t(offsets), status=status, **kw)
        assert int(status.item()) == code and torch.equal(out[0], x[0]) and torch.equal(out[1], torch.full_like(x[1], 3.0) if code else x[1])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(2, 50), (100, 20000)])
def test_histories_in_a_buffer_without_room(eng, rows, vocab):
    x = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(1)).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    tokens, total, status, out = torch.zeros((rows, 0), **i32), torch.zeros(rows, **i32), torch.zeros(1, **i32), torch.full_like(x, 3.0)
    kw = dict(out=out, tokens=tokens, prompt_lens=torch.zeros(rows, **i32), total_lens=total, frequency=torch.ones(rows, device="cuda"), status=status)
    assert torch.equal(eng.hook_adjust_logits(x, **kw), x) and int(status.item()) == 0
    total[1] = 5
    out.fill_(3.0)
    eng.hook_adjust_logits(x, **kw)
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS and (out[1] == 3.0).all() and torch.equal(out[0], x[0]) and torch.equal(out[2:], x[2:])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(3, 777), (100, 20000)])
def test_infinite_frequency_penalties(eng, rows, vocab):
    """They rule out what was generated, and nothing else: a token of the prompt or the biases was generated no times."""
    g, x, kw = _random(rows, vocab, torch.float32, 100, 17, bias=9)
    _check(eng, x, **dict(kw, freq=[float("inf")] * rows))
    _check(eng, x, **dict(kw, pres=[float("inf")] * rows))


@pytest.mark.gpu
@pytest.mark.parametrize("rep", [2.0 ** -149, 1e-40, 2.0 ** -127, 2.0 ** -126, 1e-25, 2.0 ** -64, 1.0, 2.0 ** 64, 1e25, 2.0 ** 126, 2.0 ** 127, 3.4e38])
@pytest.mark.parametrize("rows,vocab", [(2, 400), (100, 16400)])
def test_repetition_penalties_over_the_whole_range(eng, rep, rows, vocab):
    """The reciprocal and the product with it are rounded to 24 bits, powers of 2 aside: 2 x 2^-24, and a step of the numbers next to zero."""
    g = np.random.default_rng(vocab)
    x = (g.choice([-1.0, 1.0], (rows, vocab)) * np.exp2(g.uniform(-126, 127, (rows, vocab)))).astype(np.float32)
    dev = torch.from_numpy(x).cuda()
    tokens = torch.arange(vocab, dtype=torch.int32, device="cuda").expand(rows, vocab)
    lens = torch.full((rows,), vocab, dtype=torch.int32, device="cuda")
    got = eng.hook_adjust_logits(dev, out=torch.empty_like(dev), tokens=tokens, prompt_lens=lens, total_lens=lens,
                                 repetition=torch.full((rows,), rep, device="cuda")).double().cpu().numpy()
    r, x = float(np.float32(rep)), x.astype(np.float64)
    want = np.where(x > 0, x / r, x * r)
    top = float(np.finfo(np.float32).max)
    near = np.abs(np.abs(want) / top - 1) <= 2.0 ** -22             # rounded to infinity or to the largest number
    assert np.array_equal(got[(np.abs(want) > top) & ~near], np.copysign(np.inf, want[(np.abs(want) > top) & ~near]))
    fine = (np.abs(want) <= top) & ~near
    assert np.all(np.abs(got - want)[fine] <= np.abs(want[fine]) * 2.0 ** -23 + 2.0 ** -149)


@pytest.mark.gpu
def test_as_many_rows_as_there_can_be(eng):
    g, x, kw = _random(65535, 37, torch.float32, 5, 19)
    _check(eng, x, mask=g.random((3, 37)) < 0.6, mask_rows=g.integers(-1, 3, 65535).tolist(), **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab,hist", [(5, 1000, 20), (90, 20000, 20), (90, 20000, 13000)])
def test_rows_behind_the_first_4_gigabytes(eng, rows, vocab, hist):
    """Places of logits, tokens and mask words that do not fit 32 bits."""
    g, x, kw = _random(rows, vocab, torch.bfloat16, hist, 23)
    mask, i32 = g.random((rows, vocab)) < 0.6, dict(dtype=torch.int32, device="cuda")

    def far(t):
        """The same rows so far apart that the last one lies behind the first 2^32 elements."""
        step = 2 ** 32 // (rows - 1) + 9
        wide = torch.empty((rows - 1) * step + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (step, 1))
        return wide.copy_(t)

    total, prompt = (torch.tensor(kw[k], **i32) for k in ("total", "prompt"))
    rep, pres, freq = (torch.tensor(kw[k], dtype=torch.float32, device="cuda") for k in ("rep", "pres", "freq"))
    near = dict(tokens=torch.tensor(kw["tokens"], **i32), mask=_bits(mask).cuda())
    rest = dict(prompt_lens=prompt, total_lens=total, repetition=rep, presence=pres, frequency=freq)
    want = eng.hook_adjust_logits(x.cuda(), out=torch.empty(rows, vocab, device="cuda"), **near, **rest)
    assert torch.equal(eng.hook_adjust_logits(far(x.cuda()), out=far(torch.empty_like(want)), **{k: far(t) for k, t in near.items()}, **rest), want)
