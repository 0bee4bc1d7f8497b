"""A decode loop over the 4-bit cache as a program makes it: prompts appended and read back for their attention, forks, copies of shared pages, single
tokens attended over the 4-bit pages, logits edited and the next tokens drawn -- each step checked against contiguous keys and values in 64
bits that know nothing of pages."""
import numpy as np
import pytest
import torch

from oracle import ops, q4
from paper_2603_06588_b200 import binding

from .test_decode_q4 import bounds
from .test_q4_cache import _i32

HQ, HKV, D, GROUP, VOCAB, PAGES, SLOTS, WIDTH = 4, 2, 64, 32, 997, 60, 8, 8
SPANS = [[0, 5], [5, 1000]]


class Loop:
    def __init__(self):
        g = torch.Generator().manual_seed(21)
        self.eng = binding.HookAttn(0)
        self.qkv = torch.randn(VOCAB, HQ + 2 * HKV, D, generator=g).to(torch.bfloat16)          # a token's projections
        self.head = torch.randn(HQ * D, VOCAB, generator=g).cuda() / 4
        self.freq = (10000.0 ** (-torch.arange(D // 2) / (D // 2))).float().cuda()
        self.pages = torch.full((PAGES, HKV, q4.slab_bytes(D, GROUP)), 0xFF, dtype=torch.uint8, device="cuda")
        self.pool = dict(block_table=torch.full((SLOTS, WIDTH), -1, dtype=torch.int32, device="cuda"), seq_lens=_i32([0] * SLOTS),
                         page_refs=_i32([0] * PAGES), status=_i32([0]))
        self.scratch = torch.full((2, PAGES, 16, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.tokens = [[] for _ in range(SLOTS)]
        self.kv = [np.zeros((2, 0, HKV, D)) for _ in range(SLOTS)]                              # what the oracle holds: rounded to bf16, not yet quantised
        self.alpha, self.steer = torch.tensor([0.5, 0.0, -0.25, 0.0]), torch.randn(HQ, D, generator=g)

    def feed(self, new):
        """Appends new[slot] = tokens.  Returns the live slots, their tables and lengths, and the rotated queries."""
        pairs = self.eng.hook_cache_extend(**self.pool, new_rows=_i32([len(new.get(s, ())) for s in range(SLOTS)]))
        self.eng.hook_cache_copy_pages_q4([self.pages], pairs, status=self.pool["status"])
        live = sorted(new)
        rows = [t for s in live for t in new[s]]
        dev = self.qkv[rows].cuda()
        keep = dict(block_table=self.pool["block_table"][live].contiguous(), seq_lens=self.pool["seq_lens"][live].contiguous())
        cu = np.cumsum([0] + [len(new[s]) for s in live])
        q = self.eng.hook_rope_append_q4(q=dev[:, :HQ], k=dev[:, HQ:HQ + HKV], v=dev[:, HQ + HKV:], pages=self.pages, inv_freq=self.freq, cu_q_lens=_i32(cu),
                                         status=self.pool["status"], **keep)
        # the rotation itself is hook_rope_append's, whose rows the oracle takes as they are: into a bf16 cache of one page a row
        flat = torch.zeros(2, len(rows), 16, HKV, D, dtype=torch.bfloat16, device="cuda")
        at = _i32([len(self.tokens[s]) + i for s in live for i in range(len(new[s]))])
        self.eng.hook_rope_append(q=dev[:, :HQ], k=dev[:, HQ:HQ + HKV], v=dev[:, HQ + HKV:], k_cache=flat[0], v_cache=flat[1], inv_freq=self.freq,
                                  block_table=torch.arange(len(rows), device="cuda", dtype=torch.int32)[:, None], seq_lens=torch.ones_like(at),
                                  positions=at[None])
        kv = flat[:, :, 0].double().cpu().numpy()
        for i, s in enumerate(live):
            self.kv[s] = np.concatenate([self.kv[s], kv[:, cu[i]:cu[i + 1]]], axis=1)
            self.tokens[s] += new[s]
        assert self.pool["seq_lens"].tolist() == [len(t) for t in self.tokens] and int(self.pool["status"].item()) == 0
        return live, keep, cu, q

    def held(self, s, h):
        """Keys and values of a KV head as the cache stands for them: (codes, steps, lowest values)."""
        out = []
        for part in (0, 1):
            codes, step, low = q4.quantise(self.kv[s][part, :, h], GROUP)
            out.append((codes, np.repeat(step, GROUP, -1), np.repeat(low, GROUP, -1)))
        return out

    def prompt(self, new):
        """A chunk: appended, its sequences read back to bf16 pages, attended there."""
        live, keep, cu, q = self.feed(new)
        to = torch.arange(len(live) * WIDTH, device="cuda", dtype=torch.int32).view(len(live), WIDTH)
        self.eng.hook_cache_read_q4(self.pages, keep["block_table"], keep["seq_lens"], k_cache=self.scratch[0], v_cache=self.scratch[1], to_table=to,
                                    status=self.pool["status"])
        out, _ = self.eng.hook_attn_prefill(q=q, k_cache=self.scratch[0], v_cache=self.scratch[1], block_table=to, seq_lens=keep["seq_lens"], cu_q_lens=_i32(cu))
        out, q = out.double().cpu().numpy(), q.double().cpu().numpy()
        for i, s in enumerate(live):
            L = len(self.tokens[s])
            for h in range(HQ):
                (kc, ks, kl), (vc, vs, vl) = self.held(s, h // (HQ // HKV))
                k, v = q4.bf16((kc * ks + kl).astype(np.float32)), q4.bf16((vc * vs + vl).astype(np.float32))
                for r in range(cu[i], cu[i + 1]):
                    n = L - cu[i + 1] + r + 1
                    x = k[:n] @ q[r, h] / D ** 0.5
                    p = np.exp(x - x.max())
                    assert np.abs(out[r, h] - p @ v[:n] / p.sum()).max() <= 2e-2, (s, h, r)      # the attention's own tolerance

    def step(self, new):
        """One token each, over the 4-bit pages; returns the live slots and the rows' outputs."""
        live, keep, _, q = self.feed({s: [t] for s, t in new.items()})
        out, mass = self.eng.hook_attn_decode_q4(q=q, pages=self.pages, spans=_i32([SPANS] * len(live)), head_mask=torch.ones(HQ, dtype=torch.uint8),
                                                 alpha=self.alpha, steer_vec=self.steer.cuda(), status=self.pool["status"], max_seq_len=WIDTH * 16, **keep)
        got, sums, q = out.double().cpu().numpy(), mass.double().cpu().numpy(), q.double().cpu().numpy()
        for i, s in enumerate(live):
            for h in range(HQ):
                k, v = self.held(s, h // (HQ // HKV))
                want, parts, size = q4.attend(q[i, h], k, v, D ** -0.5, float(self.alpha[h]) * self.steer[h].double().numpy(), SPANS)
                most, most_mass = bounds(size, want, D)
                assert np.all(np.abs(got[i, h] - want) <= most) and np.all(np.abs(sums[i, h] - parts) <= most_mass), (s, h)
        assert int(self.pool["status"].item()) == 0
        return live, out

    def choose(self, live, out, seed):
        """The next tokens: logits edited in place, then drawn from."""
        logits = (out.float().flatten(1) @ self.head).to(torch.bfloat16)
        g = np.random.default_rng(seed)
        rows = len(live)
        width = max(len(self.tokens[s]) for s in live)
        history = _i32([self.tokens[s] + [-1] * (width - len(self.tokens[s])) for s in live])
        lens = _i32([len(self.tokens[s]) for s in live])
        edited = self.eng.hook_adjust_logits(logits, out=torch.empty(rows, VOCAB, device="cuda"), tokens=history, prompt_lens=torch.zeros_like(lens),
                                             total_lens=lens, repetition=torch.full((rows,), 1.3, device="cuda"), frequency=torch.full((rows,), 0.5, device="cuda"))
        want, scale = ops.adjust_logits(logits.double().cpu().numpy(), tokens=history.tolist(), prompt_lens=[0] * rows, total_lens=lens.tolist(),
                                        repetition=[float(np.float32(1.3))] * rows, frequency=[0.5] * rows)
        assert np.all(np.abs(edited.double().cpu().numpy() - want) <= np.abs(want) * 2.0 ** -24 + scale * 2.0 ** -21)
        args = dict(temperature=g.uniform(0.5, 1.2, rows), top_k=g.integers(1, 60, rows), top_p=g.uniform(0.5, 0.95, rows), min_p=g.uniform(0, 0.05, rows))
        u = g.random(rows).astype(np.float32)
        dev = {n: torch.tensor(v, dtype=torch.int32 if n == "top_k" else torch.float32, device="cuda") for n, v in args.items()}
        got = self.eng.hook_sample_tokens(edited, torch.from_numpy(u).cuda(), status=self.pool["status"], **dev).tolist()
        for r in range(rows):
            one = {n: int(v[r]) if n == "top_k" else float(np.float32(v[r])) for n, v in args.items()}
            token, gap = q4.sample(edited[r].double().tolist(), float(u[r]), **one)
            assert gap > 1e-10 and got[r] == token, (r, got[r], token, gap)
        return dict(zip(live, got))


@pytest.mark.gpu
def test_prompts_forks_and_sampled_steps():
    g = np.random.default_rng(22)
    loop = Loop()
    loop.prompt({0: g.integers(0, VOCAB, 37).tolist(), 1: g.integers(0, VOCAB, 16).tolist()})
    loop.prompt({0: g.integers(0, VOCAB, 5).tolist(), 2: g.integers(0, VOCAB, 3).tolist()})            # a later chunk, and a new request
    loop.eng.hook_cache_fork(**loop.pool, parents=_i32([0, 0, 1]), children=_i32([3, 4, 5]))
    for parent, child in ((0, 3), (0, 4), (1, 5)):
        loop.tokens[child], loop.kv[child] = list(loop.tokens[parent]), loop.kv[parent].copy()
    nxt = {s: int(g.integers(VOCAB)) for s in range(6)}
    for n in range(12):
        live, out = loop.step(nxt)
        nxt = loop.choose(live, out, seed=100 + n)
    loop.eng.hook_cache_free(**loop.pool, seqs=_i32([1, 4]))
    for s in (1, 4):
        loop.tokens[s], loop.kv[s] = [], np.zeros((2, 0, HKV, D))
        del nxt[s]
    for n in range(8):
        live, out = loop.step(nxt)
        nxt = loop.choose(live, out, seed=200 + n)


@pytest.mark.gpu
def test_captured_steps_beside_another_loop():
    """A whole step -- room, shared pages, append, attention, the next tokens -- in one graph that feeds itself, replayed next to eager steps of
    another pool on another stream: both hold at every step the bits of eager steps with nothing beside them."""
    eng, steps = binding.HookAttn(0), 40
    g = torch.Generator().manual_seed(31)
    qkv = torch.randn(VOCAB, HQ + 2 * HKV, D, generator=g).to(torch.bfloat16).cuda()
    head = torch.randn(HQ * D, VOCAB, generator=g).cuda() / 4
    freq = (10000.0 ** (-torch.arange(D // 2) / (D // 2))).float().cuda()
    draws = torch.rand(steps, 4, generator=g).cuda()
    heat, top = torch.tensor([0.8, 1.0, 0.0, 1.2]).cuda(), torch.tensor([0.9, 0.5, 1.0, 0.95]).cuda()

    class Pool:
        def __init__(self):
            self.pages = torch.zeros(40, HKV, q4.slab_bytes(D, GROUP), dtype=torch.uint8, device="cuda")
            self.pool = dict(block_table=torch.full((4, WIDTH), -1, dtype=torch.int32, device="cuda"), seq_lens=_i32([0] * 4),
                             page_refs=_i32([0] * 40), status=_i32([0]))
            self.tokens, self.n, self.ones = _i32([3, 5, 7, 11]), torch.zeros(1, dtype=torch.int64, device="cuda"), _i32([1] * 4)

        def step(self):
            table, lens, status = (self.pool[n] for n in ("block_table", "seq_lens", "status"))
            pairs = eng.hook_cache_extend(**self.pool, new_rows=self.ones)
            eng.hook_cache_copy_pages_q4([self.pages], pairs, status=status)
            row = qkv[self.tokens.long()]
            q = eng.hook_rope_append_q4(q=row[:, :HQ], k=row[:, HQ:HQ + HKV], v=row[:, HQ + HKV:], pages=self.pages, block_table=table, seq_lens=lens,
                                        inv_freq=freq, status=status)
            out, _ = eng.hook_attn_decode_q4(q=q, pages=self.pages, block_table=table, seq_lens=lens, status=status, max_seq_len=WIDTH * 16)
            logits = (out.float()[:, :, :, None] * head.view(HQ, D, VOCAB)).sum((1, 2))             # no workspace of a library
            eng.hook_sample_tokens(logits, draws[self.n].view(4), temperature=heat, top_p=top, tokens=self.tokens, status=status)
            self.n += 1
            return out

        def now(self, out):
            return [t.clone() for t in (out, self.tokens, self.pages, self.pool["seq_lens"], self.pool["status"])]

    alone = Pool()
    want = [alone.now(alone.step()) for _ in range(steps)]
    assert int(alone.pool["status"].item()) == 0 and alone.pool["seq_lens"].tolist() == [steps] * 4

    captured, beside, side = Pool(), Pool(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured.step()
    torch.cuda.synchronize()
    got, other = [], []
    for _ in range(steps):
        graph.replay()
        got.append(captured.now(out))
        with torch.cuda.stream(side):
            other.append(beside.now(beside.step()))
    torch.cuda.synchronize()
    for n in range(steps):
        for a, b, c in zip(want[n], got[n], other[n]):
            assert torch.equal(a, b) and torch.equal(a, c), n
