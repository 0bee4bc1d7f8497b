"""Every row of the tokens is written: filters that leave one token or ties alone, next to infinite logits and at largest logits of zero.  The
calls write into a tensor that holds what no call returns."""
import numpy as np
import pytest
import torch

from oracle import q4
from paper_2603_06588_b200 import binding

UNWRITTEN = -7


@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _draw(eng, logits, u, want=None, seen=None, **filters):
    """Tokens of the call beside ``want``, or else the oracle's of the rows ``seen`` (default: the logits); ``filters``: a value for each row."""
    rows = len(u)
    f32 = lambda a: torch.tensor(a, dtype=torch.float32, device="cuda")
    tokens, status = torch.full((rows,), UNWRITTEN, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = {n: torch.tensor(v, dtype=torch.int32, device="cuda") if n == "top_k" else f32(v) for n, v in filters.items()}
    eng.hook_sample_tokens(logits.cuda(), f32(u), tokens=tokens, status=status, **dev)
    if want is None:
        want = []
        for r in range(rows):
            one = {n: v[r] if n == "top_k" else float(np.float32(v[r])) for n, v in filters.items()}
            token, gap = q4.sample((logits if seen is None else seen)[r].double().tolist(), float(np.float32(u[r])), **one)
            assert gap > 1e-10, "choose another seed: this row is decided by rounding"
            want.append(token)
    assert tokens.tolist() == want and int(status.item()) == 0


U = [0.0, 0.99999994, 0.1234567, 0.4321]


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [5, 700, 9001, 70001, 400001])
@pytest.mark.parametrize("where", ["one", "some", "most"])
def test_no_share_next_to_infinite_logits(eng, vocab, where):
    """top_p of 0 or next to it leaves the first of the infinite logits: one, a few, or more than a warp lists; the first one is never at index 0."""
    g = np.random.default_rng(vocab)
    x = g.normal(size=(4, vocab)) * 3
    for r in range(4):
        if where == "one":
            x[r, g.integers(1, vocab)] = np.inf
        else:
            x[r, 1:][g.random(vocab - 1) < (0.01 if where == "some" else 0.9)] = np.inf
            x[r, vocab - 1 - r] = np.inf
    logits, first = torch.from_numpy(x).float(), x.argmax(1).tolist()
    for share in ([0.0] * 4, [1e-45, 1e-30, 1e-20, 0.0]):
        _draw(eng, logits, U, first, top_p=share)
        _draw(eng, logits, U, first, top_p=share, temperature=[0.3, 1.0, 1e-20, 1e20])
        _draw(eng, logits, U, first, top_p=share, min_p=[0.0, 0.5, 1.0, 1e-3])
        for k in (1, 2, vocab // 2, vocab - 1):
            _draw(eng, logits, U, first, top_p=share, top_k=[max(k, 1)] * 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_no_share_of_finite_logits(eng, dtype):
    """The same of finite rows: steep, flat, of large and of the largest values."""
    g = np.random.default_rng(5)
    most = float(torch.finfo(dtype).max)
    for vocab in (3, 4097, 33001):
        x = g.normal(size=(4, vocab))
        x[0] *= 100
        x[1] = 2.0
        x[2] = np.where(g.random(vocab) < 0.5, most, -most)
        logits = torch.from_numpy(x).to(dtype)
        first = logits.float().numpy().argmax(1).tolist()
        _draw(eng, logits, U, first, top_p=[0.0] * 4)
        _draw(eng, logits, U, first, top_p=[1e-45] * 4, top_k=[1, 2, 2, 1], temperature=[0.5] * 4)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 300, 9001, 70001])
def test_ties_at_zero(eng, dtype, vocab):
    """min_p of 1 leaves the largest logits alone, zero among them (log-probabilities whose one certain token has 0, rows of zeros of both signs).
    A weight of 1 is that of the largest alone, but 64 bits round exp(-0.5 / 1e20) = 1 - 5e-21 to it: the oracle sees the others as masked."""
    g = np.random.default_rng(vocab)
    x = -np.abs(g.normal(size=(4, vocab))) - 0.5
    x[0, vocab // 2] = 0.0
    x[1] = np.where(g.random(vocab) < 0.5, 0.0, -0.0)
    x[2, :] = -np.inf
    x[2, vocab - 1] = -0.0
    x[3][g.random(vocab) < 0.3] = 0.0
    x[3, vocab - 1] = 0.0
    logits = torch.from_numpy(x).to(dtype)
    largest = logits.masked_fill(logits < logits.amax(1, keepdim=True), -np.inf)
    one = [1.0] * 4
    for heat in (one, [0.5, 2.0, 1e-20, 1e20]):
        _draw(eng, logits, U, seen=largest, min_p=one, temperature=heat)
        _draw(eng, logits, U, seen=largest, min_p=one, temperature=heat, top_p=[0.9, 0.3, 0.0, 0.77])
        _draw(eng, logits, U, seen=largest, min_p=one, temperature=heat, top_k=[1, 3, 7, 40], top_p=[0.99] * 4)


@pytest.mark.gpu
def test_least_weights_that_end_at_zero(eng):
    """Borders of min_p and of the temperature that come to a logit of exactly zero: what lies there stays where its weight says so."""
    logits = torch.tensor([[31.0, 0.0, -1.0], [0.0, -1e-45, -1.0], [1e-45, 0.0, -1.0], [0.0, 0.0, -31.0]])
    _draw(eng, logits, [0.3, 0.6, 0.7, 0.8], temperature=[1.0] * 4)
    _draw(eng, logits, [0.3, 0.4, 0.7, 0.8], min_p=[1.0, 0.5, 0.5, 1.0], temperature=[1.0, 2.0, 1.0, 1e-30])
