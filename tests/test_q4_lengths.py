"""The longest sequences of a 4-bit cache: a table of 2^27 pages that share a few thousand, up to the last length and behind it."""
import numpy as np
import pytest
import torch

from oracle import q4
from paper_2603_06588_b200 import binding

from .test_q4_cache import _i32

D, GROUP, HQ, POOL, WIDTH, MOST = 64, 64, 2, 4096, 1 << 27, 2 ** 31 - 4096


@pytest.fixture(scope="module")
def held():
    g = np.random.default_rng(9)
    slabs = g.integers(0, 256, (POOL, 1, q4.slab_bytes(D, GROUP)), dtype=np.uint8)
    pairs = np.stack([0.2 + 0.1 * g.random((POOL, 1, 32)), -2.5 + g.random((POOL, 1, 32))], -1)
    slabs[..., 16 * D:] = torch.from_numpy(pairs).to(torch.bfloat16).view(torch.uint8).flatten(-2).numpy()
    table = (torch.arange(WIDTH, dtype=torch.int32, device="cuda") % POOL)[None]
    yield dict(eng=binding.HookAttn(0), slabs=slabs, pages=torch.from_numpy(slabs).cuda(), table=table, q=torch.from_numpy(g.normal(size=(1, HQ, D))).to(torch.bfloat16))
    torch.cuda.empty_cache()


def _attend(held, length, spans):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, mass = held["eng"].hook_attn_decode_q4(q=held["q"].cuda(), pages=held["pages"], block_table=held["table"], seq_lens=_i32([length]), spans=_i32([spans]),
                                                head_mask=torch.ones(HQ, dtype=torch.uint8), status=status)
    return out[0].double().cpu().numpy(), mass[0].double().cpu().numpy(), int(status.item())


@pytest.mark.gpu
@pytest.mark.parametrize("length", [MOST, MOST - 15, MOST - 16, MOST - 33])
def test_the_last_lengths(held, length):
    """A warp's run has some 60000 pages here.  Sums of positive 32-bit numbers, one after the other, are off by 2^-24 of them each: of 30000
    probabilities of a lane by 2^-9 at most; the matrix unit's sums, one a page, by 2^-7 at 2^-23 each.  The output's own rounding is 2^-8."""
    spans = [[0, 16], [length - 1, length], [length - 16, 2 ** 31 - 1], [length - 40, length - 16], [length // 2, length], [-5, 2 ** 31 - 1]]
    out, mass, status = _attend(held, length, spans)
    assert status == 0
    (kc, ks, kl), (vc, vs, vl) = ([x[:, 0].reshape(-1, D) for x in part] for part in q4.load(held["slabs"], D, GROUP))
    k, v = kc * ks + kl, vc * vs + vl
    times = lambda a, b: (b // (16 * POOL) - a // (16 * POOL)) + (np.arange(16 * POOL) < b % (16 * POOL)).astype(float) - (np.arange(16 * POOL) < a % (16 * POOL))
    largest = (15 * vs + np.abs(vl)).max()
    for h in range(HQ):
        x = k @ held["q"][0, h].double().numpy() * D ** -0.5
        p = np.exp(x - x.max())
        total = (p * times(0, length)).sum()
        want = (p * times(0, length)) @ v / total
        assert np.all(np.abs(out[h] - want) <= np.abs(want) * 2.0 ** -8 + largest * (2 * 2.0 ** -9 + 2.0 ** -7))
        for j, (a, b) in enumerate(spans):
            part = (p * times(max(a, 0), min(b, length))).sum() / total
            assert abs(mass[h, j] - part) <= part * 2.0 ** -7, (h, j, mass[h, j], part)      # of both sums, and of the exponentials


@pytest.mark.gpu
@pytest.mark.parametrize("length", [MOST + 1, MOST + 4000, 2 ** 31 - 17, 2 ** 31 - 1])
def test_longer_ones_are_faults(held, length):
    eng = held["eng"]
    out, mass, status = _attend(held, length, [[0, 16], [0, 2 ** 31 - 1]])
    assert status == binding.HOOK_ATTN_ERR_BOUNDS and not out.any() and not mass.any()
    cache, status = torch.full((2, POOL, 16, 1, D), 3.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    eng.hook_cache_read_q4(held["pages"], held["table"], _i32([length]), k_cache=cache[0], v_cache=cache[1], to_table=held["table"], status=status)
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS and bool((cache == 3.0).all())
    status.zero_()
    pages, row = held["pages"].clone(), torch.ones(1, 1, D, dtype=torch.bfloat16, device="cuda")
    q = eng.hook_rope_append_q4(q=row, k=row, v=row, pages=pages, block_table=held["table"], seq_lens=_i32([length]), inv_freq=torch.zeros(0, device="cuda"), status=status)
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS and not q.any() and torch.equal(pages, held["pages"])
