"""The attention over a 4-bit cache where the sizes of its values differ by much: constant groups of large values, groups of small values beside large
ones under a sharp softmax, steps that grow along the sequence.  Bounds go by the element's own group."""
import numpy as np
import pytest
import torch

from oracle import q4
from paper_2603_06588_b200 import binding

from .test_q4_cache import _i32


@pytest.fixture(scope="module")
def eng():
    return binding.HookAttn(0)


class Held:
    """One sequence of one KV head: K is 1 * code of element 0 (so a score is a whole number of q's first element), V as given."""

    def __init__(self, d, group, k_codes, v_codes, v_step, v_low, seed):
        L, g = len(k_codes), np.random.default_rng(seed)
        self.d, self.group, n = d, group, -(-L // 16)
        slabs = np.zeros((n, q4.slab_bytes(d, group)), dtype=np.uint8)
        place = {False: [q4.place_k, 0], True: [q4.place_v, 8 * d]}
        at = np.arange(L)
        for value, codes in ((False, np.pad(k_codes[:, None], ((0, 0), (0, d - 1)))), (True, v_codes)):
            find, base = place[value]
            for t in range(16):
                for e in range(d):
                    byte, high = find(t, e, d)
                    rows = at[t::16]
                    slabs[rows // 16, base + byte] |= (codes[rows, e] << (4 if high else 0)).astype(np.uint8)
        params = np.zeros((n * 16, 2, d // group, 2))
        params[:L, 0, :, 0] = 1.0
        params[:L, 1, :, 0], params[:L, 1, :, 1] = v_step, v_low
        bits = torch.from_numpy(params.reshape(n, 16, 2, -1).transpose(0, 2, 1, 3).copy()).to(torch.bfloat16)
        slabs[:, 16 * d:] = bits.reshape(n, -1).view(torch.uint8).numpy()
        self.L, self.order = L, g.permutation(n)
        self.slabs = np.zeros_like(slabs)
        self.slabs[self.order] = slabs
        k, v = q4.load(slabs[:, None], d, group)
        self.k, self.v = ([x[:, 0].reshape(-1, d)[:L] for x in part] for part in (k, v))

    def run(self, eng, q0, width, spans=None):
        """Outputs for queries that are ``q0[h]`` in element 0; ``width``: pages of the block table."""
        heads = len(q0)
        q = torch.zeros(1, heads, self.d)
        q[0, :, 0] = torch.tensor(q0)
        table = np.full((1, max(width, len(self.order))), -1)
        table[0, :len(self.order)] = self.order
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out, mass = eng.hook_attn_decode_q4(q=q.to(torch.bfloat16).cuda(), pages=torch.from_numpy(self.slabs[:, None].copy()).cuda(), block_table=_i32(table),
                                            seq_lens=_i32([self.L]), scale=1.0, status=status, spans=None if spans is None else _i32([spans]),
                                            head_mask=None if spans is None else torch.ones(heads, dtype=torch.uint8))
        assert int(status.item()) == 0
        return out[0].double().cpu().numpy(), None if mass is None else mass[0].double().cpu().numpy()

    def check(self, eng, q0, width, spans=None):
        """Of each element: the output's rounding to bf16 (2^-8); probabilities times steps as halves, off by 2^-11, and those that are subnormal
        there by 2^-25 where the group's largest step is at least 2^6 and the largest probability 1; probabilities off by what 32 bits leave
        of the scores on either side (2^-23 of sums of d + 8 terms, the exponential's 2^-21), for values up to the element's largest; and
        32-bit sums in 64 pieces."""
        out, mass = self.run(eng, q0, width, spans)
        _, vs, vl = self.v
        largest = np.abs(15 * vs + np.abs(vl)).max(0)
        for h, a in enumerate(q0):
            q = np.zeros(self.d)
            q[0] = a
            want, sums, size = q4.attend(q, self.k, self.v, 1.0, 0.0, [] if spans is None else spans)
            off = 2 * size["x"] * (self.d + 8) * 2.0 ** -23 + 2.0 ** -21
            most = np.abs(want) * 2.0 ** -8 + size["coded"] * 2.0 ** -11 + self.L * 15 * vs.max(0) * 2.0 ** -31 + (2 * off + 64 * 2.0 ** -22) * largest
            assert np.all(np.abs(out[h] - want) <= most), (h, np.abs(out[h] - want).max(), most.max())
            if spans is not None:
                assert np.all(np.abs(mass[h] - sums) <= 2 * off + 2.0 ** -18), (h, mass[h], sums)


WIDTHS = [0, 40000]                    # chunks; shares of the pages


@pytest.mark.gpu
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("d,group", [(64, 64), (64, 32), (128, 32), (128, 64), (128, 128)])
@pytest.mark.parametrize("power", [39, 60, 100, -100])
def test_constant_groups_of_any_size(eng, d, group, power, width):
    """Groups without a step hold their value exactly, up to sizes whose sum over the keys still fits 32 bits, of either sign."""
    g = np.random.default_rng(power + 200)
    L, n = 1500, d // group
    low = 2.0 ** power * g.uniform(1, 2, (L, n)) * np.where(g.random((L, n)) < 0.5, -1, 1)
    held = Held(d, group, g.integers(0, 16, L), np.zeros((L, d), dtype=np.int64), np.zeros((L, n)), low, seed=1)
    held.check(eng, [1.0, -0.5, 0.0], width, [[0, 700], [699, 1500]])
    low[:, 0] = 2.0 ** power                                   # the same in all tokens
    Held(d, group, g.integers(0, 16, L), np.zeros((L, d), dtype=np.int64), np.zeros((L, n)), low, seed=2).check(eng, [1.0, 0.25], width)


@pytest.mark.gpu
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("d,group", [(64, 32), (128, 32), (128, 64)])
@pytest.mark.parametrize("ratio", [-4, -8, -10, -14, -24, -60])
@pytest.mark.parametrize("sharp", [0, 20001])
def test_small_groups_beside_large_ones(eng, d, group, ratio, sharp, width):
    """One token holds most of the probability (12 above the others' scores) and has codes 0; the others' codes are what is left to see.  Each group's steps
    are 2^ratio of the group before it, or, in the last of four, none."""
    g = np.random.default_rng(ratio + 100)
    L, n = 32768, d // group
    k, v = np.zeros(L, dtype=np.int64), g.integers(8, 16, (L, d))
    k[sharp], v[sharp] = 12, 0
    step = 2.0 ** (ratio * np.arange(n)) * g.uniform(1, 2, (L, n))
    if n == 4:
        step[:, 3] = 0
    low = -3 * step
    held = Held(d, group, k, v, step, low, seed=3)
    held.check(eng, [1.0, 0.875, 0.0, -1.0], width, [[0, 100], [100, 32768], [20001, 20002]])


@pytest.mark.gpu
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 128)])
@pytest.mark.parametrize("kind", ["growing", "falling", "mixed", "largest"])
def test_steps_along_the_sequence(eng, d, group, kind, width):
    """A group's steps from 2^-60 to 2^3 (or up to 2^109, where the sums still fit 32 bits), growing with the tokens, falling or in no order, each group at its own pace."""
    g = np.random.default_rng(11)
    L, n = 2000, d // group
    at = np.linspace(0, 1, L)[:, None] * np.ones(n) if kind != "mixed" else g.random((L, n))
    if kind == "falling":
        at = at[::-1]
    power = 3 - 63 * (1 - at) / (1 + np.arange(n)) if kind != "largest" else 108 - 40 * at * np.arange(n)
    step = 2.0 ** np.round(power) * g.uniform(1, 2, (L, n)) * (g.random((L, n)) < 0.9)
    low = -8 * step
    held = Held(d, group, g.integers(0, 4, L), g.integers(0, 16, (L, d)), step, low, seed=4)
    held.check(eng, [1.0, 0.5, 0.0, 2.0, -1.0], width, [[0, 16], [31, 33], [1000, 5000]])
