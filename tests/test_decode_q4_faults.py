"""The rows of a page out of range over a 4-bit cache, beside pages that read as NaN or whose scores are infinite."""
import pytest
import torch

from paper_2603_06588_b200 import binding

from .test_decode_q4 import Case


@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


@pytest.mark.gpu
@pytest.mark.parametrize("width", [0, 40000])
@pytest.mark.parametrize("kind", ["keys", "values", "scores"])
@pytest.mark.parametrize("bad,odd", [(6, 1), (1, 6), (20, 3), (3, 20), (40, 41), (43, 0)])
def test_nothing_is_left_of_a_broken_row(eng, bad, odd, kind, width):
    """A page out of range and one whose keys or values are NaN, or whose keys are so large that scores overflow, in one warp's run, in two of a chunk,
    in two chunks: outputs and span masses of that row are zeros, and the other rows are as they were."""
    c = Case([700, 700], 8, 2, 128, 128, spans=3, steer=True, width=width, q_size=64.0 if kind == "scores" else 1.0)
    c.mask[:] = 1
    good = eng.hook_attn_decode_q4(**c.kw())
    kw = c.kw()
    pages, kw["block_table"] = c.pages.clone(), kw["block_table"].clone()
    at = 16 * 128 + (16 * 4 if kind == "values" else 0)
    pair = [0, 0, 0x7F, 0x7F] if kind == "scores" else [0xFF] * 4                 # lowest 3.4e38; NaN
    pages[int(c.table[0, odd]), :, at:at + 16 * 4] = torch.tensor(pair * 16, dtype=torch.uint8, device="cuda")
    kw["block_table"][0, bad] = len(c.slabs)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, mass = eng.hook_attn_decode_q4(**{**kw, "pages": pages, "status": status})
    assert int(status.item()) == binding.HOOK_ATTN_ERR_BOUNDS
    assert torch.equal(out[0], torch.zeros_like(out[0])) and torch.equal(mass[0], torch.zeros_like(mass[0]))
    assert torch.equal(out[1], good[0][1]) and torch.equal(mass[1], good[1][1])


@pytest.mark.gpu
@pytest.mark.parametrize("width", [0, 40000])
def test_infinite_scores_are_not_hidden(eng, width):
    """Keys of 3.4e38: heads whose query adds up to more than 0 have scores of +infinity and read as NaN, the others pass over those keys."""
    c = Case([700, 33], 8, 2, 128, 128, width=width, q_size=64.0)
    pages = c.pages.clone()
    pages[int(c.table[0, 1]), :, 16 * 128:16 * 128 + 16 * 4] = torch.tensor([0, 0, 0x7F, 0x7F] * 16, dtype=torch.uint8, device="cuda")
    out, _ = eng.hook_attn_decode_q4(**{**c.kw(), "pages": pages})
    sums = c.q[0].double().sum(1)
    assert (sums.abs() > 12).all()                          # 12 x 3.39e38 / sqrt(128) is more than 32 bits hold, in units of ln 2 as well
    for h in range(8):
        assert torch.isnan(out[0, h]).all() if sums[h] > 0 else torch.isfinite(out[0, h]).all()
    assert torch.isfinite(out[1]).all()
