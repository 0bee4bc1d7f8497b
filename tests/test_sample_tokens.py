"""The choice of a token: oracle pins, refusals (CPU) and GPU parity, token by token."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import q4
from paper_2603_06588_b200 import binding

from ._ops import FAKE_HANDLE, no_device, struct_fields

INVALID, UNSUPPORTED = binding.HOOK_ATTN_ERR_INVALID_ARG, binding.HOOK_ATTN_ERR_UNSUPPORTED


# --------------------------------------------------------------------------------------------------- CPU
def test_struct_mirror():
    assert struct_fields("hook_sample_params") == [f[0] for f in binding.HookSampleParams._fields_]


def test_oracle_filters():
    x = [1.0, 3.0, 2.0, 3.0, 0.0, -math.inf, math.nan]
    kept = lambda **kw: q4.kept(x, **{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **kw})[0]
    assert kept() == [0, 1, 2, 3, 4]
    assert kept(temperature=0) == [1]
    assert kept(top_k=1) == [1] and kept(top_k=2) == [1, 3] and kept(top_k=3) == [1, 2, 3] and kept(top_k=7) == kept(top_k=-1) == kept()
    assert kept(min_p=1.0) == [1, 3] and kept(min_p=math.exp(-1) * 0.999) == [1, 2, 3]
    total = 2 + math.exp(-1) + math.exp(-2) + math.exp(-3)
    assert kept(top_p=0.0) == [1] and kept(top_p=0.99 / total) == [1] and kept(top_p=1.01 / total) == [1, 3] and kept(top_p=2.01 / total) == [1, 2, 3]
    assert kept(top_k=3, top_p=0.9) == [1, 2, 3] and kept(top_k=3, top_p=0.8) == [1, 3]      # of the three's weight
    assert q4.kept([math.inf, 5.0, math.inf], 1.0, 0, 1.0, 0.0)[1] == [1.0, 0.0, 1.0]


def test_oracle_draws():
    x = [0.0, math.log(2.0), math.log(5.0)]
    assert [q4.sample(x, u)[0] for u in (0.0, 0.12, 0.13, 0.37, 0.38, 0.999)] == [0, 0, 1, 1, 2, 2]
    assert abs(q4.sample(x, 0.25)[1] - 0.125) < 1e-12


def _params(**over):
    p = binding.HookSampleParams()
    p.num_rows, p.vocab_size, p.logits_row_stride = 2, 1000, 1000
    p.logits = p.uniform = p.tokens = 0x10000
    for k, v in over.items():
        setattr(p, k, v)
    return p


@no_device
@pytest.mark.parametrize("over,code", [
    (dict(), binding.HOOK_ATTN_ERR_CUDA), (dict(num_rows=0, logits=None), binding.HOOK_ATTN_ERR_CUDA), (dict(logits_row_stride=0), binding.HOOK_ATTN_ERR_CUDA),
    (dict(num_rows=-1), INVALID), (dict(vocab_size=0), INVALID), (dict(dtype=3), INVALID), (dict(logits=None), INVALID), (dict(uniform=None), INVALID),
    (dict(tokens=None), INVALID), (dict(logits_row_stride=-1), INVALID), (dict(vocab_size=2 ** 20 + 1), UNSUPPORTED), (dict(num_rows=65536), UNSUPPORTED),
    (dict(logits=0x10001), UNSUPPORTED), (dict(logits=0x10002, dtype=binding.HOOK_DTYPE_F32), UNSUPPORTED)])
def test_refusals(over, code):
    assert binding.load_library().hook_sample_tokens(FAKE_HANDLE, ctypes.byref(_params(**over)), None) == code


def test_no_handle_and_no_params():
    lib = binding.load_library()
    assert lib.hook_sample_tokens(None, ctypes.byref(_params()), None) == INVALID
    assert lib.hook_sample_tokens(None, None, None) == INVALID


# --------------------------------------------------------------------------------------------------- GPU
@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _f32(a):
    return torch.tensor(a, dtype=torch.float32, device="cuda")


def _check(eng, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, dev=None):
    """Every row's token is the oracle's; no random number may lie so near a border that 64-bit sums could differ about it."""
    rows = len(u)
    dev = logits.cuda() if dev is None else dev
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    opt = lambda a, t: None if a is None else torch.tensor(a, dtype=t, device="cuda")
    got = eng.hook_sample_tokens(dev, _f32(u), temperature=opt(temperature, torch.float32), top_k=opt(top_k, torch.int32), top_p=opt(top_p, torch.float32),
                                 min_p=opt(min_p, torch.float32), status=status)
    single = lambda a, r, default: default if a is None else float(np.float32(a[r]))
    for r in range(rows):
        want, gap = q4.sample(logits[r].double().tolist(), float(np.float32(u[r])), single(temperature, r, 1.0), 0 if top_k is None else top_k[r],
                              single(top_p, r, 1.0), single(min_p, r, 0.0))
        assert gap > 1e-10, "choose another seed: this row is decided by rounding"
        assert int(got[r]) == want, (r, int(got[r]), want)
    assert int(status.item()) == 0
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 4096, 4097, 20011, 65537])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_parity(eng, vocab, dtype):
    """Each filter alone, all together, none; 16-bit types bring ties."""
    g = np.random.default_rng(vocab)
    rows = 7
    logits = torch.from_numpy(g.normal(size=(rows, vocab)) * 3).to(dtype)
    u = [0.0, 0.999999] + g.random(rows - 2).tolist()
    heat = (0.3 + 1.2 * g.random(rows)).tolist()
    k = [1, 2, 5, 50, 700, 0, vocab - 1]
    p = [0.0, 0.3, 0.6, 0.9, 0.95, 0.999, 1.0]
    least = [0.0, 1.0, 0.5, 0.1, 0.02, 0.001, 0.3]
    _check(eng, logits, u)
    _check(eng, logits, u, temperature=heat)
    _check(eng, logits, u, top_k=k)
    _check(eng, logits, u, temperature=heat, top_p=p)
    _check(eng, logits, u, temperature=heat, min_p=least)
    _check(eng, logits, u, temperature=[0.0, 1.0] * 3 + [0.0], top_k=k[::-1], top_p=p, min_p=least[::-1])
    _check(eng, logits, u, temperature=heat, top_k=k[::-1], top_p=p)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["constant", "two values", "steep", "shifted", "tiny", "wide", "masked", "one left", "infinite", "zeros"])
def test_rows_of_a_kind(eng, kind):
    g = np.random.default_rng(3)
    vocab, rows = 9001, 6
    x = g.normal(size=(rows, vocab))
    if kind == "constant":
        x[:] = -2.5
    elif kind == "two values":
        x = np.where(x > 1.5, 4.0, 3.0)
    elif kind == "steep":
        x *= 100
    elif kind == "shifted":
        x += 1e4
    elif kind == "tiny":
        x *= 1e-30
    elif kind == "wide":
        x *= 3e37
    elif kind == "masked":
        x[g.random(x.shape) < 0.99] = -np.inf
        x[0, ::7] = np.nan
    elif kind == "one left":
        x[:] = -np.inf
        x[np.arange(rows), [0, 1, 4500, 8999, 9000, 77]] = -3e38
    elif kind == "infinite":
        x[:, ::3000] = np.inf
    elif kind == "zeros":
        x = np.where(g.random(x.shape) < 0.5, 0.0, -0.0)
    logits = torch.from_numpy(x).float()
    u = [0.0, 0.99999994, 0.1234567, 0.4321, 0.7654321, 0.5000123]
    _check(eng, logits, u)
    _check(eng, logits, u, temperature=[0.7, 0.0, 1.5, 1e-3, 40.0, 1e30], top_k=[3, 0, 4000, 9000, 2500, 1])
    _check(eng, logits, u, top_p=[0.31, 0.0, 0.7, 0.999, 0.5, 0.12345])
    _check(eng, logits, u, temperature=[0.9] * 6, top_k=[2, 50, 900, 8000, 0, 5], top_p=[0.61, 0.33, 0.501, 0.999, 0.17, 0.9], min_p=[0, 0, 0.01, 0, 0, 0.9])


@pytest.mark.gpu
def test_extreme_temperatures(eng):
    """From a temperature at which only ties are left to one at which all finite logits weigh the same, with and without an infinite one."""
    g = np.random.default_rng(7)
    x = g.normal(size=(6, 3001)) * 4
    x[:, ::500] = np.round(x[:, ::500])
    heat = [1e-44, 1e-20, 1e-6, 1e20, 1.5e37, 3.4e38]
    u = g.random(6).tolist()
    logits = torch.from_numpy(x).float()
    for more in (dict(), dict(top_k=[40] * 6), dict(top_p=[0.77] * 6), dict(min_p=[0.3] * 6)):
        _check(eng, logits, u, temperature=heat, **more)
    logits[:, 700], logits[:, 2000] = float("inf"), float("inf")
    for more in (dict(), dict(top_k=[2] * 6), dict(top_p=[0.77] * 6), dict(min_p=[0.3] * 6)):
        _check(eng, logits, u, temperature=heat, **more)


@pytest.mark.gpu
def test_strides_alignment_and_outputs(eng):
    """Rows that start anywhere, padded rows, one row for all, a tensor of their own for the tokens."""
    g = np.random.default_rng(4)
    flat = torch.from_numpy(g.normal(size=50021) * 2)
    u = g.random(5).tolist()
    for dtype in (torch.bfloat16, torch.float32):
        base = flat.to(dtype)
        for vocab, stride, offset in ((5001, 5001, 1), (4999, 6007, 3), (6007, 6007, 5), (9, 11, 7), (5000, 0, 2)):
            view = lambda b: torch.as_strided(b, (5, vocab), (stride, 1), offset)
            _check(eng, view(base), u, top_k=[0, 20, 300, 1, 2], top_p=[0.9] * 5, dev=view(base.cuda()))
    logits, tokens = torch.from_numpy(g.normal(size=(5, 100))).float().cuda(), torch.full((5,), 9, dtype=torch.int32, device="cuda")
    got = eng.hook_sample_tokens(logits, _f32(u), tokens=tokens)
    assert got.data_ptr() == tokens.data_ptr() and torch.equal(tokens, eng.hook_sample_tokens(logits, _f32(u)))
    assert eng.hook_sample_tokens(logits[:0], _f32([])).shape == (0,)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,vocab", [(1, 160000), (2, 2 ** 20), (300, 700), (3, 392001), (150, 21000)])
def test_large_calls(eng, rows, vocab):
    """A vocabulary that a cluster cannot hold, and more rows than SMs."""
    g = np.random.default_rng(rows)
    logits = torch.from_numpy(g.normal(size=(rows, vocab)) * 2).float()
    u = g.random(rows).tolist()
    _check(eng, logits, u, top_p=g.uniform(0.5, 0.99, rows).tolist())
    _check(eng, logits, u, temperature=[0.8] * rows, top_k=g.integers(1, 600, rows).tolist(), min_p=[0.01] * rows)


@pytest.mark.gpu
def test_faults(eng):
    """Rows without a choice or with parameters out of range get -1 and set status; the others are drawn as ever."""
    x = torch.randn(6, 300, generator=torch.Generator().manual_seed(5))
    x[1], x[2] = -math.inf, math.nan
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    u = [0.3, 0.3, 0.3, 0.4, 0.5, 0.6]
    got = eng.hook_sample_tokens(x.cuda(), _f32(u), status=status).tolist()
    assert got[1] == got[2] == -1 and int(status.item()) == INVALID
    assert [got[r] for r in (0, 3, 4, 5)] == [q4.sample(x[r].double().tolist(), float(np.float32(u[r])))[0] for r in (0, 3, 4, 5)]
    good = dict(temperature=[1.0] * 6, top_p=[0.9] * 6, min_p=[0.1] * 6, uniform=u)
    for name, bad in (("uniform", 1.0), ("uniform", -0.1), ("uniform", math.nan), ("temperature", -1.0), ("temperature", math.inf), ("temperature", math.nan),
                      ("top_p", -0.1), ("top_p", math.nan), ("min_p", 1.5), ("min_p", -0.5), ("min_p", math.nan)):
        args = {k: list(v) for k, v in good.items()}
        args[name][4] = bad
        status.zero_()
        out = eng.hook_sample_tokens(x.cuda(), _f32(args.pop("uniform")), status=status, **{k: _f32(v) for k, v in args.items()}).tolist()
        assert out[4] == -1 and int(status.item()) == INVALID and out[0] >= 0 and out[3] >= 0 and out[5] >= 0


@pytest.mark.gpu
def test_graphs_and_streams(eng):
    g = np.random.default_rng(6)
    logits, u = torch.from_numpy(g.normal(size=(9, 30011)) * 3).float().cuda(), _f32(g.random(9).tolist())
    kw = dict(temperature=_f32([0.8] * 9), top_k=torch.full((9,), 90, dtype=torch.int32, device="cuda"), top_p=_f32([0.9] * 9))
    want = eng.hook_sample_tokens(logits, u, **kw)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = eng.hook_sample_tokens(logits, u, stream=side.cuda_stream, **kw)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = eng.hook_sample_tokens(logits, u, **kw)
    for _ in range(3):
        captured.fill_(-5)
        graph.replay()
        assert torch.equal(captured, want)
    u.copy_(1 - u)                                          # a replay reads what is there by then
    graph.replay()
    assert torch.equal(captured, eng.hook_sample_tokens(logits, u, **kw))


@pytest.mark.gpu
def test_refused_tensors(eng):
    x, u = torch.zeros(2, 50, device="cuda"), _f32([0.1, 0.2])
    for bad in (dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.T), dict(logits=x.cpu()), dict(uniform=u[:1]), dict(uniform=u.double()),
                dict(temperature=u.half()), dict(top_k=u), dict(top_p=u[:1]), dict(min_p=u.cpu()), dict(tokens=u)):
        args = {**dict(logits=x, uniform=u), **bad}
        with pytest.raises(AssertionError):
            eng.hook_sample_tokens(args.pop("logits"), args.pop("uniform"), **args)
