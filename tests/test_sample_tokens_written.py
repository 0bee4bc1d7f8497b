"""Every row of the tokens is written: filters that leave one token alone, next to infinite logits too.  The calls write into a tensor that holds what no call returns."""
import numpy as np
import pytest
import torch

from paper_2603_06588_b200 import binding

UNWRITTEN = -7


@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


def _draw(eng, logits, u, want, **filters):
    """Tokens of the call beside ``want``; ``filters``: a value for each row."""
    rows = len(u)
    f32 = lambda a: torch.tensor(a, dtype=torch.float32, device="cuda")
    tokens, status = torch.full((rows,), UNWRITTEN, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = {n: torch.tensor(v, dtype=torch.int32, device="cuda") if n == "top_k" else f32(v) for n, v in filters.items()}
    eng.hook_sample_tokens(logits.cuda(), f32(u), tokens=tokens, status=status, **dev)
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
