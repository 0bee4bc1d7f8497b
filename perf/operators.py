"""Operators of a decode loop around the hooked paged attention, as cases that can be timed and compared.

Three groups: rotary positions with several axes that append their keys and values to the paged cache, the
pages of that cache (fork, extend, free, compact, copy), and the edits of the logits that follow (penalties for
repeated tokens, biases, grammar masks).  With ``own`` false ``run`` computes them from elementary torch
operations; with ``own`` true it makes the calls of the library.
"""
import numpy as np
import torch

own = False

PAGE = 16                     # tokens per page: the library's page size
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_library = None


def library():
    """The library's binding and its handle, made once like in a serving program."""
    global _library
    if _library is None:
        from paper_2603_06588_b200 import binding
        _library = binding, binding.HookAttn(0)
    return _library


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one sequence in an interactive chat: a step is all latency
        dict(name="rope decode 1", op="rope", seqs=1, rows=1, decode=True, ctx_lo=4096, ctx_hi=4096, hq=32, hkv=8, d=128, rot=128,
             sections="64", order="blocked", pairing="halves", dtype="bf16", far=0, given=False),
        # a full decode batch
        dict(name="rope decode 256", op="rope", seqs=256, rows=256, decode=True, ctx_lo=64, ctx_hi=2048, hq=28, hkv=4, d=128, rot=128,
             sections="16,24,24", order="blocked", pairing="halves", dtype="bf16", far=0, given=True),
        # packed prompts of uneven lengths in 32 bits: a partial rotation of neighbouring elements, far positions
        dict(name="rope ragged fp32", op="rope", seqs=37, rows=5003, decode=False, ctx_lo=0, ctx_hi=700, hq=8, hkv=8, d=64, rot=40,
             sections="8,6,6", order="cyclic", pairing="adjacent", dtype="fp32", far=1000000, given=True),
        # four long prompts with images
        dict(name="rope prompt 65536", op="rope", seqs=4, rows=65536, decode=False, ctx_lo=0, ctx_hi=100, hq=64, hkv=8, d=128, rot=128,
             sections="24,20,20", order="cyclic", pairing="halves", dtype="bf16", far=0, given=True),
        # one chat turn, a small vocabulary
        dict(name="logits 1 x 32000", op="logits", rows=1, vocab=32000, dtype="bf16", out="fp32", history=300, bias=0, grammar=False),
        # odd vocabulary, odd number of rows, everything on, rounded back to fp16
        dict(name="logits 7 x 50001", op="logits", rows=7, vocab=50001, dtype="fp16", out="fp16", history=2500, bias=100, grammar=True),
        # a decode batch with long histories
        dict(name="logits 64 x 128000", op="logits", rows=64, vocab=128000, dtype="bf16", out="fp32", history=32768, bias=300, grammar=True),
        # the largest batch, 32-bit logits
        dict(name="logits 256 x 160000", op="logits", rows=256, vocab=160000, dtype="fp32", out="fp32", history=4096, bias=16, grammar=True),
        # one request sampled four times, one layer's cache at a time
        dict(name="branch 1 x 4", op="branch", parents=1, branches=4, new=1, lo=100, hi=3000, layers=1, hkv=8, d=128),
        # a batch of requests sampled eight times, drafts of five tokens, the caches of all layers
        dict(name="branch 32 x 8", op="branch", parents=32, branches=8, new=5, lo=100, hi=700, layers=16, hkv=8, d=128),
        # a small pool, one layer
        dict(name="compact 700", op="compact", pages=700, fill=0.5, seqs=24, shared=0.25, layers=1, hkv=4, d=64),
        # a fragmented pool before its tail is given back
        dict(name="compact 4096", op="compact", pages=4096, fill=0.6, seqs=64, shared=0.25, layers=16, hkv=8, d=128),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["rope", "rope", "logits", "logits", "branch", "compact"])
    if op == "rope":
        d = rng.choice([64, 128])
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.randint(1, 8)
        rot = rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)])
        pairs = rot // 2
        axes = rng.choice([1, 3, 3, 2, 4]) if pairs >= 4 else 1
        cuts = sorted(rng.randint(0, pairs) for _ in range(axes - 1))
        sections = ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [pairs]))
        decode = rng.random() < 0.4
        rows = _log(rng, 1, 512) if decode else _log(rng, 16, 65536)
        ctx = _log(rng, 1, 2048)
        return dict(op=op, seqs=rows if decode else min(rows, _log(rng, 1, 64)), rows=rows, decode=decode, ctx_lo=ctx // 2, ctx_hi=ctx,
                    hq=hq, hkv=hkv, d=d, rot=rot, sections=sections, order=rng.choice(["blocked", "cyclic"]),
                    pairing=rng.choice(["halves", "adjacent"]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    far=rng.choice([0, 0, 1000000]), given=axes > 1 or rng.random() < 0.5)
    if op == "logits":
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        return dict(op=op, rows=_log(rng, 1, 256), vocab=_log(rng, 1000, 160000), dtype=dtype, out=rng.choice([dtype, "fp32"]),
                    history=_log(rng, 1, 8192), bias=rng.choice([0, 1, 30, 300]), grammar=rng.random() < 0.6)
    if op == "branch":
        return dict(op=op, parents=_log(rng, 1, 32), branches=rng.randint(1, 8), new=rng.choice([1, 1, 2, 5, 17, 40]), lo=1, hi=_log(rng, 16, 700),
                    layers=rng.randint(1, 16), hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]))
    return dict(op=op, pages=_log(rng, 64, 4096), fill=0.2 + 0.7 * rng.random(), seqs=rng.randint(1, 64), shared=0.5 * rng.random(),
                layers=rng.randint(1, 16), hkv=rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128]))


# ----------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    host = np.random.default_rng(seed)
    dev = torch.Generator(device="cuda")
    dev.manual_seed(int(seed))
    make = {"rope": _prepare_rope, "logits": _prepare_logits, "branch": _prepare_branch, "compact": _prepare_compact}[case["op"]]
    return dict(case=dict(case), **make(case, host, dev))


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def _randn(dev, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda", dtype=dtype, generator=dev)


def _sections(case):
    return [int(x) for x in case["sections"].split(",")]


def _axis_of_pair(case):
    """The axis whose position turns each pair: blocks of pairs one after the other, or dealt out in turn to the axes that still have some left."""
    left, axes = _sections(case), []
    if case["order"] == "blocked":
        return [a for a, n in enumerate(left) for _ in range(n)]
    while any(left):
        for a in range(len(left)):
            if left[a]:
                axes.append(a)
                left[a] -= 1
    return axes


def _prepare_rope(case, host, dev):
    seqs, rows, hq, hkv, d = (case[k] for k in ("seqs", "rows", "hq", "hkv", "d"))
    if case["decode"]:
        n = np.ones(seqs, dtype=np.int64)
    else:
        cuts = np.sort(host.integers(0, rows + 1, seqs - 1))
        n = np.diff(np.concatenate([[0], cuts, [rows]]))
    lens = n + host.integers(case["ctx_lo"], case["ctx_hi"] + 1, seqs)
    pages = -(-lens // PAGE)
    pool = seqs * (-(-case["ctx_hi"] // PAGE) + 1) + rows // PAGE + 1
    order = host.permutation(pool)
    table = np.full((seqs, -(-(rows // (seqs if case["decode"] else 1) + case["ctx_hi"]) // PAGE)), -1, dtype=np.int64)
    table[np.arange(table.shape[1]) < pages[:, None]] = order[:pages.sum()]
    row_pos = np.concatenate([np.arange(l - m, l) for l, m in zip(lens, n)]) + case["far"]
    # text, with an image of 24 x 32 patches in every 1024 tokens: (time, height, width), and a fourth axis that counts images
    at = row_pos % 1024
    image = at >= 256
    t = np.where(image, row_pos - at + 256, row_pos)
    grid = [t, np.where(image, t + (at - 256) // 32, t), np.where(image, t + (at - 256) % 32, t), row_pos // 1024]
    axes = len(_sections(case))
    dt = DTYPES[case["dtype"]]
    qkv = _randn(dev, rows, hq + 2 * hkv, d, dtype=dt)          # what a fused projection leaves
    cache = _randn(dev, pool, 2, PAGE, hkv, d)
    freq = (10000.0 if axes == 1 else 1000000.0) ** -(np.arange(case["rot"] // 2) * 2.0 / max(1, case["rot"]))
    return dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], k_cache=cache[:, 0], v_cache=cache[:, 1], cache=cache,
                block_table=_dev(table), seq_lens=_dev(lens), cu_q_lens=None if case["decode"] else _dev(np.concatenate([[0], np.cumsum(n)])),
                positions=_dev(np.stack(grid[:axes])) if case["given"] else None, inv_freq=_dev(freq, torch.float32),
                axis_pairs=_sections(case), factor=1.0 if axes == 1 else 1.25)


def _prepare_logits(case, host, dev):
    rows, vocab, hist = case["rows"], case["vocab"], case["history"]
    total = host.integers(1, hist + 1, rows)
    total[0] = hist
    prompt = (total * host.random(rows)).astype(np.int64)
    u = torch.rand(rows, hist, device="cuda", generator=dev)     # few tokens come often, most seldom
    tokens = (u.pow(4) * vocab).long().clamp_(max=vocab - 1).int()
    tokens[torch.arange(hist, device="cuda") >= _dev(total)[:, None]] = -1
    state = dict(logits=_randn(dev, rows, vocab, dtype=torch.float32).mul_(3).to(DTYPES[case["dtype"]]), tokens=tokens, prompt_lens=_dev(prompt),
                 total_lens=_dev(total), repetition=_dev(1 + 0.3 * host.random(rows), torch.float32),
                 presence=_dev(host.random(rows), torch.float32), frequency=_dev(0.5 * host.random(rows), torch.float32),
                 bias=None, mask=None, mask_rows=None)
    if case["bias"]:
        counts = host.integers(0, case["bias"] + 1, rows)
        counts[0] = case["bias"]
        step = vocab // case["bias"]
        picks = [host.permutation(case["bias"])[:c] * step + host.integers(0, step, c) for c in counts]   # no token twice in a row
        state["bias"] = (_dev(np.concatenate([[0], np.cumsum(counts)])), _dev(np.concatenate(picks)),
                         _dev(host.normal(size=int(counts.sum())) * 5, torch.float32))
    if case["grammar"]:
        words = -(-vocab // 32)
        which = np.where(host.random(rows) < 0.75, np.arange(rows), -1)            # the other requests have no grammar
        which[0] = 0
        bits = [torch.randint(-2 ** 31, 2 ** 31, (rows, words), device="cuda", generator=dev, dtype=torch.int64).int() for _ in range(3)]
        state["mask"] = bits[0] & bits[1] | bits[2] & bits[0]
        state["mask_rows"] = _dev(which)
    return state


def _caches(case, pool, dev):
    caches = _randn(dev, case["layers"], 2, pool, PAGE, case["hkv"], case["d"])
    return dict(caches=caches, layers=[(c[0], c[1]) for c in caches])


def _prepare_branch(case, host, dev):
    parents, branches = case["parents"], case["branches"]
    lens = host.integers(case["lo"], case["hi"] + 1, parents)
    pages = -(-lens // PAGE)
    longest = -(-(case["hi"] + case["new"]) // PAGE)
    pool = parents * longest + parents * branches * (-(-case["new"] // PAGE) + 1)
    seqs = parents * (1 + branches)
    table = np.full((seqs, longest), -1, dtype=np.int64)
    table[:parents][np.arange(table.shape[1]) < pages[:, None]] = host.permutation(pool)[:pages.sum()]
    refs = np.zeros(pool, dtype=np.int64)
    refs[table[table >= 0]] = 1
    new = np.zeros(seqs, dtype=np.int64)
    new[parents:] = case["new"]
    return dict(block_table=_dev(table), seq_lens=_dev(np.concatenate([lens, np.zeros(seqs - parents)])), page_refs=_dev(refs),
                parents=_dev(np.repeat(np.arange(parents), branches)), children=_dev(np.arange(parents, seqs)), new_rows=_dev(new),
                **_caches(case, pool, dev))


def _prepare_compact(case, host, dev):
    pool, seqs = case["pages"], case["seqs"]
    used = max(1, int(pool * case["fill"]))
    pages = host.permutation(pool)[:used]
    share = np.full(seqs, used // seqs)
    more = host.integers(0, used // seqs + 1, seqs // 2)                          # long sequences and short ones
    share[:seqs // 2] += more
    share[seqs - seqs // 2:] -= more
    share[0] += used % seqs
    forked = (share * case["shared"]).astype(np.int64)                            # a fork of each sequence that holds its first pages
    table = np.full((2 * seqs, 2 * (used // seqs) + used % seqs), -1, dtype=np.int64)
    at = np.arange(table.shape[1])
    table[:seqs][at < share[:, None]] = pages
    table[seqs:] = np.where(at < forked[:, None], table[:seqs], -1)
    counts = np.concatenate([share, forked])
    lens = np.maximum(0, counts * PAGE - host.integers(0, PAGE, 2 * seqs) * (counts > 0))
    refs = np.zeros(pool, dtype=np.int64)
    np.add.at(refs, table[table >= 0], 1)
    return dict(block_table=_dev(table), seq_lens=_dev(lens), page_refs=_dev(refs), **_caches(case, pool, dev))


# ------------------------------------------------------------------------------------------- one pass
def run(state):
    return {"rope": _run_rope, "logits": _run_logits, "branch": _run_branch, "compact": _run_compact}[state["case"]["op"]](state)


def _run_rope(s):
    case = s["case"]
    if own:
        lib, eng = library()
        q_out = eng.hook_rope_append(
            q=s["q"], k=s["k"], v=s["v"], k_cache=s["k_cache"], v_cache=s["v_cache"], block_table=s["block_table"], seq_lens=s["seq_lens"],
            cu_q_lens=s["cu_q_lens"], positions=s["positions"], inv_freq=s["inv_freq"], axis_pairs=s["axis_pairs"],
            axis_order=lib.HOOK_ROPE_AXES_CYCLIC if case["order"] == "cyclic" else lib.HOOK_ROPE_AXES_BLOCKED,
            pairing=lib.HOOK_ROPE_PAIR_HALVES if case["pairing"] == "halves" else lib.HOOK_ROPE_PAIR_ADJACENT, factor=s["factor"])
        return [q_out, s["cache"]]
    rows = torch.arange(case["rows"], device="cuda")
    lens = s["seq_lens"].long()
    if s["cu_q_lens"] is None:
        seq, at = rows, lens - 1
    else:
        cu = s["cu_q_lens"].long()
        seq = torch.searchsorted(cu, rows, right=True) - 1
        at = lens[seq] - cu[seq + 1] + rows
    pos = s["positions"].double() if s["positions"] is not None else at.double().expand(len(s["axis_pairs"]), -1)
    axis = torch.tensor(_axis_of_pair(case), device="cuda", dtype=torch.long)
    angle = pos[axis].T * s["inv_freq"].double()                                   # [rows, pairs]
    cos, sin = ((f(angle) * s["factor"]).float()[:, None] for f in (torch.cos, torch.sin))
    q_out = torch.empty(s["q"].shape, dtype=torch.bfloat16, device="cuda")
    q_out.copy_(_rotate(s["q"].float(), cos, sin, case))
    page, slot = s["block_table"].long()[seq, at // PAGE], at % PAGE
    s["k_cache"][page, slot] = _rotate(s["k"].float(), cos, sin, case).bfloat16()
    s["v_cache"][page, slot] = s["v"].bfloat16()
    return [q_out, s["cache"]]


def _rotate(x, cos, sin, case):
    rot = case["rot"]
    if case["pairing"] == "halves":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _run_logits(s):
    case = s["case"]
    rows, vocab = s["logits"].shape
    out = torch.empty(rows, vocab, dtype=DTYPES[case["out"]], device="cuda")
    if own:
        offsets, bias_tokens, bias_values = s["bias"] or (None, None, None)
        library()[1].hook_adjust_logits(
            s["logits"], out=out, tokens=s["tokens"], prompt_lens=s["prompt_lens"], total_lens=s["total_lens"], repetition=s["repetition"],
            presence=s["presence"], frequency=s["frequency"], bias_offsets=offsets, bias_tokens=bias_tokens, bias_values=bias_values,
            mask=s["mask"], mask_rows=s["mask_rows"])
        return out
    x = s["logits"].float()
    at = torch.arange(s["tokens"].shape[1], device="cuda")
    live = at < s["total_lens"][:, None]
    made = live & (at >= s["prompt_lens"][:, None])
    tokens = s["tokens"].long().clamp(0, vocab - 1)
    seen = torch.zeros(rows, vocab, device="cuda").scatter_add_(1, tokens, live.float()) > 0
    count = torch.zeros(rows, vocab, device="cuda").scatter_add_(1, tokens, made.float())
    rep = s["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias"] is not None:
        offsets, bias_tokens, bias_values = s["bias"]
        entry = torch.arange(bias_tokens.numel(), device="cuda")
        row = torch.searchsorted(offsets.long(), entry, right=True) - 1
        x[row, bias_tokens.long()] += bias_values
    if s["mask"] is not None:
        bit = torch.arange(vocab, device="cuda")
        words = s["mask"][s["mask_rows"].clamp(min=0).long()]
        allowed = (words[:, bit // 32] >> (bit % 32).int()) & 1
        x = torch.where((allowed == 0) & (s["mask_rows"] >= 0)[:, None], float("-inf"), x)
    out.copy_(x)
    return out


def _run_branch(s):
    """A step of sampling one prompt several times: the last step's branches go, new ones are made, get room for their tokens, and the
    pages that they would share while writing are copied."""
    table, lens, refs = s["block_table"], s["seq_lens"], s["page_refs"]
    if own:
        eng = library()[1]
        pool = dict(block_table=table, seq_lens=lens, page_refs=refs)
        eng.hook_cache_free(**pool, seqs=s["children"])
        eng.hook_cache_fork(**pool, parents=s["parents"], children=s["children"])
        pairs = eng.hook_cache_extend(**pool, new_rows=s["new_rows"])
        eng.hook_cache_copy_pages(s["layers"], pairs)
        return [table, lens, refs, pairs, s["caches"]]
    parents, children, new = s["parents"].long(), s["children"].long(), s["new_rows"]
    old = table[children]
    refs.index_add_(0, old.clamp(min=0).flatten().long(), -(old >= 0).int().flatten())
    table[children], lens[children] = -1, 0
    taken = table[parents]
    table[children], lens[children] = taken, lens[parents]
    refs.index_add_(0, taken.clamp(min=0).flatten().long(), (taken >= 0).int().flatten())
    have, want = (lens + PAGE - 1) // PAGE, (lens + new + PAGE - 1) // PAGE
    seq = torch.arange(lens.numel(), device="cuda")
    last = table[seq, (have - 1).clamp(min=0).long()]
    split = (new > 0) & (lens % PAGE != 0) & (refs[last.clamp(min=0).long()] > 1)
    need = want - have + split.int()
    first = torch.cumsum(need, 0) - need
    free = torch.argsort((refs > 0).int(), stable=True).int()
    j = torch.arange(table.shape[1], device="cuda")
    row, nth = torch.nonzero(j < need[:, None], as_tuple=True)
    page = free[first[row] + nth]
    table[row, (have - split.int()).long()[row] + nth] = page
    refs[page.long()] = 1
    refs.index_add_(0, last.clamp(min=0).long(), -split.int())
    lens += new
    pairs = torch.where(split[:, None], torch.stack([last, free[first.clamp(max=free.numel() - 1).long()]], 1), -1)
    live = pairs[pairs[:, 0] >= 0].long()
    s["caches"][:, :, live[:, 1]] = s["caches"][:, :, live[:, 0]]
    return [table, lens, refs, pairs, s["caches"]]


def _run_compact(s):
    table, lens, refs = s["block_table"], s["seq_lens"], s["page_refs"]
    if own:
        eng = library()[1]
        new_table, new_refs, page_map, pairs, num_pairs = eng.hook_cache_compact(block_table=table, seq_lens=lens, page_refs=refs)
        eng.hook_cache_copy_pages(s["layers"], pairs, num_pairs=num_pairs)
        return [new_table, new_refs, page_map, pairs, num_pairs, s["caches"]]
    used = refs > 0
    page = torch.arange(refs.numel(), device="cuda")
    low = page < used.sum()
    source, hole = page[used & ~low], page[~used & low]
    page_map = torch.where(used, page, -1).int()
    page_map[source] = hole.int()
    inside = torch.arange(table.shape[1], device="cuda") < ((lens + PAGE - 1) // PAGE)[:, None]
    new_table = torch.where(inside, page_map[table.clamp(min=0).long()], -1)
    new_refs = torch.zeros_like(refs)
    new_refs[page_map[used].long()] = refs[used]
    pairs = torch.full((refs.numel() // 2, 2), -1, dtype=torch.int32, device="cuda")
    pairs[:source.numel()] = torch.stack([source, hole], 1).int()
    num_pairs = (used & ~low).sum(dtype=torch.int32).reshape(1)
    s["caches"][:, :, hole] = s["caches"][:, :, source]
    return [new_table, new_refs, page_map, pairs, num_pairs, s["caches"]]


# ------------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "rope":
        size = 4 if case["dtype"] == "fp32" else 2
        values = case["rows"] * (case["hq"] + 2 * case["hkv"]) * case["d"]
        turned = case["rows"] * (case["hq"] + case["hkv"]) * case["rot"]
        return dict(bytes=values * (size + 2) + case["rows"] * 4 * len(_sections(case)) * case["given"], flops=turned * 3)
    if case["op"] == "logits":
        size = sum(2 if case[k] != "fp32" else 4 for k in ("dtype", "out"))
        values = case["rows"] * case["vocab"]
        grammar = values / 8 * 0.75 if case["grammar"] else 0
        return dict(bytes=values * size + grammar + case["rows"] * (case["history"] / 2 * 4 + case["bias"] / 2 * 8), flops=values)
    slab = case["layers"] * 2 * PAGE * case["hkv"] * case["d"] * 2
    if case["op"] == "branch":
        kids = case["parents"] * case["branches"]
        pages = (case["lo"] + case["hi"]) / 2 / PAGE                   # a child's table: taken back, and written anew from its parent's
        split = kids * (1 - 1 / PAGE if case["hi"] > 1 else 1)
        return dict(bytes=2 * split * slab + kids * pages * 4 * 3 + case["parents"] * pages * 4, flops=0)
    moved = case["pages"] * case["fill"] * (1 - case["fill"])
    return dict(bytes=2 * moved * slab + case["pages"] * 4 * 3 + case["pages"] * case["fill"] * 4 * 2, flops=0)


# ---------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"rope": _exact_rope, "logits": _exact_logits, "branch": _exact_branch, "compact": _exact_compact}[case["op"]](state, case)


def _exact_rope(s, case):
    """Each pair as a complex number, multiplied by exp(i * position * frequency)."""
    lens = s["seq_lens"].tolist()
    cu = s["cu_q_lens"].tolist() if s["cu_q_lens"] is not None else list(range(len(lens) + 1))
    place = [(q, lens[q] - (cu[q + 1] - cu[q]) + i) for q in range(len(lens)) for i in range(cu[q + 1] - cu[q])]
    seq, at = (torch.tensor(x, device="cuda") for x in zip(*place))
    rot = case["rot"]
    angle = torch.empty(case["rows"], rot // 2, dtype=torch.float64, device="cuda")
    for i, a in enumerate(_axis_of_pair(case)):
        angle[:, i] = (at if s["positions"] is None else s["positions"][a]).double() * s["inv_freq"][i].double()
    turn = torch.polar(torch.full_like(angle, s["factor"]), angle)[:, None]

    def turned(x):
        y = x.double()
        halves = case["pairing"] == "halves"
        re, im = (y[..., :rot // 2], y[..., rot // 2:rot]) if halves else (y[..., 0:rot:2], y[..., 1:rot:2])
        z = torch.complex(re, im) * turn
        if halves:
            y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
        else:
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        return y

    cache = s["cache"].double()
    where = s["block_table"][seq, torch.div(at, PAGE, rounding_mode="floor")].long() * PAGE + at % PAGE
    pages, _, _, hkv, d = cache.shape
    for part, rows in ((0, turned(s["k"])), (1, s["v"].double())):
        flat = cache[:, part].reshape(pages * PAGE, hkv, d)
        flat[where] = rows
        cache[:, part] = flat.view(pages, PAGE, hkv, d)
    return [turned(s["q"]), cache]


def _exact_logits(s, case):
    x = s["logits"].double().cpu().numpy()
    tokens, prompt, total = (s[k].cpu().numpy() for k in ("tokens", "prompt_lens", "total_lens"))
    rep, pres, freq = (s[k].double().cpu().numpy() for k in ("repetition", "presence", "frequency"))
    bias = [t.cpu().numpy() for t in s["bias"]] if s["bias"] else None
    for r in range(case["rows"]):
        seen = np.unique(tokens[r, :total[r]])
        x[r, seen] = np.where(x[r, seen] > 0, x[r, seen] / rep[r], x[r, seen] * rep[r])
        made, count = np.unique(tokens[r, prompt[r]:total[r]], return_counts=True)
        x[r, made] -= freq[r] * count + pres[r]
        if bias:
            lo, hi = bias[0][r], bias[0][r + 1]
            x[r, bias[1][lo:hi]] += bias[2][lo:hi].astype(np.float64)
        if s["mask"] is not None and (m := int(s["mask_rows"][r])) >= 0:
            bits = np.unpackbits(s["mask"][m].cpu().numpy().view(np.uint8), bitorder="little")[:case["vocab"]]
            x[r, bits == 0] = -np.inf
    return torch.from_numpy(x)


def _exact_branch(s, case):
    """Only the copied values: the rest are whole numbers."""
    lens, table, refs = s["seq_lens"].tolist(), s["block_table"].tolist(), s["page_refs"].tolist()
    free = [p for p, n in enumerate(refs) if n == 0]
    caches = s["caches"].float()
    for parent, child in zip(s["parents"].tolist(), s["children"].tolist()):
        have = -(-lens[parent] // PAGE)
        split = lens[parent] % PAGE != 0
        if split:
            caches[:, :, free[0]] = caches[:, :, table[parent][have - 1]]
        free = free[-(-(lens[parent] + case["new"]) // PAGE) - have + split:]
    return [None, None, None, None, caches]


def _exact_compact(s, case):
    refs = s["page_refs"].tolist()
    used = sum(n > 0 for n in refs)
    source = [p for p, n in enumerate(refs) if n > 0 and p >= used]
    hole = [p for p, n in enumerate(refs) if n == 0 and p < used]
    caches = s["caches"].float()
    for a, b in zip(source, hole):
        caches[:, :, b] = caches[:, :, a]
    return [None, None, None, None, None, caches]
