"""The calls around the attention as a decode loop makes them: prompts, forks, drafts, a compaction, eviction -- each step checked against
contiguous keys and values in 64 bits that know nothing of pages.  And the same calls on another stream, in a graph, and on a handle
whose device is not current."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import ops
from paper_2603_06588_b200 import binding

HQ, HKV, D, VOCAB = 4, 2, 64, 997
SECTIONS = (12, 10, 10)
TOL_OUT, TOL_MASS = 2e-2, 1e-3                   # the attention's own tolerances


class Sequence:
    """What the oracle knows of a sequence: its tokens and its rounded keys and values."""

    def __init__(self, tokens=(), k=None, v=None, prompt=0):
        self.tokens, self.prompt = list(tokens), prompt
        self.k = np.zeros((0, HKV, D)) if k is None else k
        self.v = np.zeros((0, HKV, D)) if v is None else v

    def fork(self):
        return Sequence(self.tokens, self.k.copy(), self.v.copy(), self.prompt)


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def _attend(q, seq, steer, alpha, spans):
    """One query row per head over all keys of the sequence."""
    out, mass = np.zeros((HQ, D)), np.zeros((HQ, len(spans)))
    for h in range(HQ):
        x = seq.k[:, h // (HQ // HKV)] @ q[h] / np.sqrt(D)
        p = np.exp(x - x.max())
        p /= p.sum()
        out[h] = p @ seq.v[:, h // (HQ // HKV)] + alpha[h] * steer[h]
        mass[h] = [p[a:b].sum() for a, b in spans]
    return out, mass


class Loop:
    def __init__(self, layers=2):
        g = torch.Generator().manual_seed(5)
        self.eng = binding.HookAttn(0)
        self.table_qkv = torch.randn(layers, VOCAB, HQ + 2 * HKV, D, generator=g).to(torch.bfloat16)      # a token's projections, layer by layer
        self.head = torch.randn(HQ * D, VOCAB, generator=g).cuda() / 16
        self.freq = (10000.0 ** (-torch.arange(32) / 32)).float()
        self.slots, self.width, self.pages, self.layers = 12, 12, 90, layers
        i32 = lambda *s, fill=0: torch.full(s, fill, dtype=torch.int32, device="cuda")
        self.pool = dict(block_table=i32(self.slots, self.width, fill=-1), seq_lens=i32(self.slots), page_refs=i32(self.pages), status=i32(1))
        self.caches = [tuple(torch.full((self.pages, 16, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv") for _ in range(layers)]
        self.seqs = [[Sequence() for _ in range(layers)] for _ in range(self.slots)]
        self.steer = torch.randn(HQ, D, generator=g)
        self.alpha = torch.tensor([0.5, 0.0, -0.25, 0.0])
        self.spans = torch.tensor([[0, 5], [5, 1000]], dtype=torch.int32)

    def i32(self, a):
        return torch.tensor(a, dtype=torch.int32, device="cuda")

    def positions(self, rows):
        """(time, height, width) of each row: text, and a picture in every second block of eight."""
        p = [[t, t + t % 3, t + t % 5] if t // 8 % 2 else [t] * 3 for _, t in rows]
        return np.ascontiguousarray(np.array(p).reshape(-1, 3).T)

    def feed(self, new, decode):
        """Appends new[slot] = tokens and attends; returns the outputs of the last layer, row by row."""
        grow = [len(new.get(s, ())) for s in range(self.slots)]
        pairs = self.eng.hook_cache_extend(**self.pool, new_rows=self.i32(grow))
        self.eng.hook_cache_copy_pages(self.caches, pairs, status=self.pool["status"])
        live = sorted(new)
        rows = [(s, len(self.seqs[s][0].tokens) + i) for s in live for i in range(len(new[s]))]
        tokens = [t for s in live for t in new[s]]
        pos = self.positions(rows)
        keep = dict(block_table=self.pool["block_table"][live].contiguous(), seq_lens=self.pool["seq_lens"][live].contiguous())
        if not decode:
            keep["cu_q_lens"] = self.i32(np.cumsum([0] + [len(new[s]) for s in live]))
        outs = []
        for l in range(self.layers):
            qkv = self.table_qkv[l][tokens]
            dev = qkv.cuda()
            k_cache, v_cache = self.caches[l]
            q = self.eng.hook_rope_append(q=dev[:, :HQ], k=dev[:, HQ:HQ + HKV], v=dev[:, HQ + HKV:], k_cache=k_cache, v_cache=v_cache,
                                          inv_freq=self.freq.cuda(), positions=self.i32(pos), axis_pairs=SECTIONS,
                                          axis_order=binding.HOOK_ROPE_AXES_CYCLIC, status=self.pool["status"], **keep)
            attend = self.eng.hook_attn_decode if decode else self.eng.hook_attn_prefill
            out, mass = attend(q=q, k_cache=k_cache, v_cache=v_cache, spans=self.spans.cuda().expand(len(live), 2, 2).contiguous(),
                               head_mask=torch.ones(HQ, dtype=torch.uint8), steer_vec=self.steer.cuda(), alpha=self.alpha, **keep)
            want = qkv.double().numpy()
            want, _ = ops.rotate(want, pos, self.freq.double().numpy(), SECTIONS, True, False, 1.0)
            for r, (s, _) in enumerate(rows):
                seq = self.seqs[s][l]
                seq.tokens.append(tokens[r])
                seq.k = np.concatenate([seq.k, _bf16(want[r:r + 1, HQ:HQ + HKV])])
                seq.v = np.concatenate([seq.v, qkv[r:r + 1, HQ + HKV:].double().numpy()])
                ref, ref_mass = _attend(_bf16(want[r, :HQ]), seq, self.steer.double().numpy(), self.alpha.tolist(), self.spans.tolist())
                assert np.abs(out[r].double().cpu().numpy() - ref).max() <= TOL_OUT, (s, l, r)
                assert np.abs(mass[r].double().cpu().numpy() - ref_mass).max() <= TOL_MASS, (s, l, r)
            outs.append(out)
        assert self.pool["seq_lens"].tolist() == [len(q[0].tokens) for q in self.seqs]
        assert int(self.pool["status"].item()) == 0
        return live, outs[-1]

    def choose(self, live, out, mask):
        """The next token of each row: the logits edited, the largest taken."""
        logits = out.float().flatten(1) @ self.head
        seqs = [self.seqs[s][0] for s in live]
        width = max(len(q.tokens) for q in seqs)
        tokens = [q.tokens + [-1] * (width - len(q.tokens)) for q in seqs]
        rows = len(live)
        ones = lambda v: torch.full((rows,), v, device="cuda")
        words = torch.from_numpy(np.packbits(np.pad(mask, ((0, 0), (0, -VOCAB % 32))), axis=1, bitorder="little").view(np.int32).copy()).cuda()
        got = self.eng.hook_adjust_logits(logits.to(torch.bfloat16), out=torch.empty_like(logits), tokens=self.i32(tokens),
                                          prompt_lens=self.i32([q.prompt for q in seqs]), total_lens=self.i32([len(q.tokens) for q in seqs]),
                                          repetition=ones(1.3), presence=ones(0.2), frequency=ones(0.7), mask=words,
                                          mask_rows=self.i32([r % 2 for r in range(rows)]), status=self.pool["status"])
        want, scale = ops.adjust_logits(logits.to(torch.bfloat16).double().cpu().numpy(), tokens=tokens, prompt_lens=[q.prompt for q in seqs],
                                        total_lens=[len(q.tokens) for q in seqs], repetition=[float(np.float32(1.3))] * rows,
                                        presence=[float(np.float32(0.2))] * rows, frequency=[float(np.float32(0.7))] * rows, mask=mask,
                                        mask_rows=[r % 2 for r in range(rows)])
        res = got.double().cpu().numpy()
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(res), fine) and np.all(np.abs(res[fine] - want[fine]) <= np.abs(want[fine]) * 2.0 ** -24 + scale[fine] * 2.0 ** -21)
        return {s: [t] for s, t in zip(live, got.argmax(1).tolist())}


@pytest.mark.gpu
def test_decode_loop_with_forks_compaction_and_eviction():
    g = np.random.default_rng(8)
    loop = Loop()
    mask = g.random((2, VOCAB)) < 0.5
    prompts = {0: g.integers(0, VOCAB, 33).tolist(), 1: g.integers(0, VOCAB, 16).tolist(), 2: g.integers(0, VOCAB, 5).tolist()}
    loop.feed(prompts, decode=False)
    for s, p in prompts.items():
        for q in loop.seqs[s]:
            q.prompt = len(p)
    # each prompt three times: 33 tokens end inside a page, 16 with one
    parents, children = [0, 0, 0, 1, 1, 1, 2, 2], [3, 4, 5, 6, 7, 8, 9, 10]
    loop.eng.hook_cache_fork(**loop.pool, parents=loop.i32(parents), children=loop.i32(children))
    for a, b in zip(parents, children):
        loop.seqs[b] = [q.fork() for q in loop.seqs[a]]
    step = {s: [int(t)] for s, t in zip(range(11), g.integers(0, VOCAB, 11))}
    for i in range(6):
        live, out = loop.feed(step, decode=True)
        step = loop.choose(live, out, mask)
        if i == 2:                                # two branches go, one falls back to its first 18 tokens, what is left moves together
            keep = [0, 0, 18]
            loop.eng.hook_cache_free(**loop.pool, seqs=loop.i32([4, 7, 3]), keep_lens=loop.i32(keep))
            for s, n in zip([4, 7, 3], keep):
                for q in loop.seqs[s]:
                    q.tokens, q.k, q.v, q.prompt = q.tokens[:n], q.k[:n], q.v[:n], min(q.prompt, n)
            step = {s: t for s, t in step.items() if s not in (4, 7)}
            pool = {k: v for k, v in loop.pool.items() if k != "status"}
            table, refs, _, pairs, count = loop.eng.hook_cache_compact(**pool, status=loop.pool["status"])
            loop.eng.hook_cache_copy_pages(loop.caches, pairs, num_pairs=count, status=loop.pool["status"])
            loop.pool.update(block_table=table, page_refs=refs)
            used = int((refs > 0).sum())
            assert (refs[:used] > 0).all() and not refs[used:].any()
            for c in loop.caches:                 # the tail is given back: nothing may read it any more
                for t in c:
                    t[used:] = float("nan")
    # a draft of four tokens for everybody
    loop.feed({s: g.integers(0, VOCAB, 4).tolist() for s in step}, decode=False)
    loop.eng.hook_cache_free(**loop.pool, seqs=loop.i32(list(range(loop.slots))))
    assert not loop.pool["page_refs"].any() and not loop.pool["seq_lens"].any() and (loop.pool["block_table"] == -1).all()
    assert int(loop.pool["status"].item()) == 0


def _one_step(eng, state, stream=None):
    """A fork, the room, the copies, an append and an edit; all of it on one stream."""
    pool = dict(block_table=state["table"], seq_lens=state["lens"], page_refs=state["refs"])
    eng.hook_cache_free(**pool, seqs=state["children"], stream=stream)
    eng.hook_cache_fork(**pool, parents=state["parents"], children=state["children"], stream=stream)
    pairs = eng.hook_cache_extend(**pool, new_rows=state["new"], stream=stream)
    eng.hook_cache_copy_pages([(state["k_cache"], state["v_cache"])], pairs, stream=stream)
    q = eng.hook_rope_append(q=state["q"], k=state["k"], v=state["v"], k_cache=state["k_cache"], v_cache=state["v_cache"], block_table=state["table"][2:],
                             seq_lens=state["lens"][2:], inv_freq=state["freq"], stream=stream)
    moved = eng.hook_cache_compact(**pool, stream=stream)
    logits = eng.hook_adjust_logits(state["logits"], out=state["edited"], tokens=state["tokens"], prompt_lens=state["prompt"], total_lens=state["total"],
                                    frequency=state["strength"], mask=state["mask"], stream=stream)
    return [pairs, q, logits, *moved, state["table"], state["lens"], state["refs"], state["k_cache"], state["v_cache"]]


def _state(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    rn = lambda *s, dt=torch.bfloat16: torch.randn(*s, generator=g, device="cuda").to(dt)
    table = torch.full((6, 4), -1, dtype=torch.int32, device="cuda")
    table[0, :3], table[1, :1] = i32([40, 7, 30]), i32([3])
    refs = torch.zeros(50, dtype=torch.int32, device="cuda")
    refs[[40, 7, 30, 3]] = 1
    return dict(table=table, lens=i32([37, 16, 0, 0, 0, 0]), refs=refs, parents=i32([0, 0, 1, 1]), children=i32([2, 3, 4, 5]), new=i32([0, 0, 1, 1, 1, 1]),
                k_cache=rn(50, 16, 2, 64), v_cache=rn(50, 16, 2, 64), q=rn(4, 4, 64), k=rn(4, 2, 64), v=rn(4, 2, 64), freq=rn(32, dt=torch.float32).abs(),
                logits=rn(4, 5000, dt=torch.float32), edited=torch.empty(4, 5000, device="cuda"), tokens=torch.randint(0, 5000, (4, 300), generator=g, device="cuda").int(),
                prompt=i32([0, 5, 300, 100]), total=i32([300, 5, 300, 200]), strength=rn(4, dt=torch.float32),
                mask=torch.randint(-2 ** 31, 2 ** 31 - 1, (4, 157), generator=g, device="cuda").int())


def _same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.gpu
def test_another_stream_and_a_graph():
    eng = binding.HookAttn(0)
    want = [t.clone() for t in _one_step(eng, _state(1))]
    again = _state(1)
    _one_step(eng, again)
    assert _same(_one_step(eng, again), want)     # the branches of the last step go first: the step can be repeated

    side, state = torch.cuda.Stream(), _state(1)
    torch.cuda.synchronize()
    got = _one_step(eng, state, stream=side.cuda_stream)
    side.synchronize()
    assert _same(got, want)

    state = _state(1)
    graph = torch.cuda.CUDAGraph()
    _one_step(eng, state)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = _one_step(eng, state)
    fresh = _state(2)
    for name, t in state.items():                 # new data, and the pool as it was at first
        t.copy_(fresh[name])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert _same(got, _one_step(eng, _state(2)))


@pytest.mark.gpu
def test_two_streams_at_once():
    """Two threads' worth of work on two streams share nothing but the handle."""
    eng = binding.HookAttn(0)
    want = [[t.clone() for t in _one_step(eng, _state(s))] for s in (3, 4)]
    streams, states = [torch.cuda.Stream() for _ in range(2)], [_state(s) for s in (3, 4)]
    torch.cuda.synchronize()
    for _ in range(20):
        got = [_one_step(eng, st, stream=s.cuda_stream) for st, s in zip(states, streams)]
    torch.cuda.synchronize()
    assert _same(got[0], want[0]) and _same(got[1], want[1])


@pytest.mark.gpu
def test_the_handles_device_must_be_current():
    """As for the other entry points: the test edits the ordinal that the handle remembers (its first field)."""
    eng, state = binding.HookAttn(0), _state(1)
    _one_step(eng, state)
    field = ctypes.cast(eng._h, ctypes.POINTER(ctypes.c_int))
    assert field[0] == 0
    field[0] = 1
    pool = dict(block_table=state["table"], seq_lens=state["lens"], page_refs=state["refs"])
    pairs = torch.full((6, 2), -1, dtype=torch.int32, device="cuda")
    calls = [lambda: eng.hook_cache_free(**pool, seqs=state["children"]), lambda: eng.hook_cache_fork(**pool, parents=state["parents"], children=state["children"]),
             lambda: eng.hook_cache_extend(**pool, new_rows=state["new"]), lambda: eng.hook_cache_compact(**pool),
             lambda: eng.hook_cache_copy_pages([(state["k_cache"], state["v_cache"])], pairs), lambda: eng.hook_adjust_logits(state["logits"]),
             lambda: eng.hook_rope_append(q=state["q"], k=state["k"], v=state["v"], k_cache=state["k_cache"], v_cache=state["v_cache"],
                                          block_table=state["table"][2:], seq_lens=state["lens"][2:], inv_freq=state["freq"])]
    try:
        for call in calls:
            with pytest.raises(binding.HookAttnError) as e:
                call()
            assert e.value.code == binding.HOOK_ATTN_ERR_INVALID_ARG
    finally:
        field[0] = 0
    torch.cuda.synchronize()
