"""Operators of a decode loop over a cache held in 4 bits, as cases that can be timed and compared.

Four groups: new rows quantised as they are written and the cache read back to bf16 pages (what a chunk of a prompt needs before its
attention), the hooked attention of single query rows over the 4-bit pages, copies of such pages, and the choice of a token from the
logits.  With ``own`` false ``run`` computes them from elementary torch operations; with ``own`` true it makes the calls of the library.

A page of one KV head is a slab of bytes: the codes of the keys (16 tokens), those of the values, and for each token and group of a head's
elements the pair (step, lowest value) in bf16, keys first.  An element is lowest + step * code.
"""
import numpy as np
import torch

own = False

PAGE = 16                     # tokens per page: the library's page size
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_library = None


def library():
    """The library's handle, made once like in a serving program."""
    global _library
    if _library is None:
        from paper_2603_06588_b200 import binding
        _library = binding.HookAttn(0)
    return _library


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token of a chat, kept in 4 bits, and its short context read back: all latency
        dict(name="store 1", op="store", seqs=1, rows=1, decode=True, ctx_lo=300, ctx_hi=300, hq=32, hkv=8, d=128, rot=128, group=128, dtype="bf16"),
        # chunks of uneven prompts in 32 bits, a partial rotation, small heads in two groups each
        dict(name="store ragged fp32", op="store", seqs=37, rows=5003, decode=False, ctx_lo=0, ctx_hi=700, hq=8, hkv=4, d=64, rot=40, group=32, dtype="fp32"),
        # four long prompts, four groups to a head
        dict(name="store prompt 65536", op="store", seqs=4, rows=65536, decode=False, ctx_lo=0, ctx_hi=4096, hq=64, hkv=8, d=128, rot=128, group=32,
             dtype="bf16"),
        # one chat, no probes
        dict(name="attend 1 x 2000", op="attend", seqs=1, lo=2000, hi=2000, hq=32, hkv=8, d=128, group=128, spans=0, probed=0, steer=False),
        # small heads, odd numbers of sequences and of heads, two spans on some heads, sequences from one token on
        dict(name="attend 37 ragged", op="attend", seqs=37, lo=1, hi=3001, hq=15, hkv=3, d=64, group=32, spans=2, probed=7, steer=True),
        # four long contexts, every head probed over eight spans
        dict(name="attend 4 x 32768", op="attend", seqs=4, lo=32768, hi=32768, hq=64, hkv=8, d=128, group=32, spans=8, probed=64, steer=True),
        # a full decode batch
        dict(name="attend 256 x 8192", op="attend", seqs=256, lo=1024, hi=8192, hq=28, hkv=4, d=128, group=64, spans=4, probed=14, steer=True),
        # the pages that forked sequences write into, all layers
        dict(name="copy 256", op="copy", pages=1024, pairs=256, layers=16, hkv=8, d=128, group=64),
        # one request's fork, one layer
        dict(name="copy 3", op="copy", pages=64, pairs=3, layers=1, hkv=4, d=64, group=32),
        # one chat turn, a small vocabulary
        dict(name="sample 1 x 32000", op="sample", rows=1, vocab=32000, dtype="bf16", filters="all"),
        # odd sizes, the whole distribution
        dict(name="sample 7 x 50001", op="sample", rows=7, vocab=50001, dtype="fp16", filters="none"),
        # the largest batch, 32-bit logits, each row with its own filters
        dict(name="sample 256 x 160000", op="sample", rows=256, vocab=160000, dtype="fp32", filters="all"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["store", "store", "store", "attend", "attend", "attend", "sample", "sample", "sample", "copy"])
    d = rng.choice([64, 128, 128])
    group = rng.choice([g for g in (32, 64, 128) if g <= d])
    hkv = rng.choice([1, 2, 3, 4, 8])
    hq = hkv * rng.randint(1, 8)
    if op == "store":
        decode = rng.random() < 0.4
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rows = _log(rng, 1, 512) if decode else _log(rng, 16, 32768 if dtype == "fp32" else 65536)
        seqs = rows if decode else min(rows, _log(rng, 1, 64))
        ctx = min(_log(rng, 1, 4096), 32768 // seqs)
        return dict(op=op, seqs=seqs, rows=rows, decode=decode, ctx_lo=ctx // 2, ctx_hi=ctx, hq=hq, hkv=hkv, d=d,
                    rot=rng.choice([0, d, d, 2 * rng.randint(1, d // 2)]), group=group, dtype=dtype)
    if op == "attend":
        seqs = _log(rng, 1, 256)
        hi = min(_log(rng, 1, 32768), 4194304 // (seqs * hkv))
        spans = rng.choice([0, 2, 3, 4, 8])
        return dict(op=op, seqs=seqs, lo=rng.choice([1, hi, hi // 2 + 1]), hi=hi, hq=hq, hkv=hkv, d=d, group=group, spans=spans,
                    probed=rng.randint(1, hq) if spans else 0, steer=rng.random() < 0.5)
    if op == "sample":
        return dict(op=op, rows=_log(rng, 1, 256), vocab=_log(rng, 1000, 160000), dtype=rng.choice(["bf16", "fp16", "fp32"]),
                    filters=rng.choice(["all", "all", "top_k", "top_p", "min_p", "none"]))
    pages = _log(rng, 16, 1024)
    return dict(op=op, pages=pages, pairs=rng.randint(1, pages // 2), layers=rng.randint(1, 7), hkv=hkv, d=d, group=group)


# ----------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    host = np.random.default_rng(seed)
    dev = torch.Generator(device="cuda")
    dev.manual_seed(int(seed))
    make = {"store": _prepare_store, "attend": _prepare_attend, "copy": _prepare_copy, "sample": _prepare_sample}[case["op"]]
    return dict(case=dict(case), **make(case, host, dev))


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).cuda()


def _randn(dev, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, device="cuda", dtype=dtype, generator=dev)


def slab_bytes(case):
    return PAGE * case["d"] + 8 * PAGE * (case["d"] // case["group"])


def _slabs(case, shape, dev):
    """Pages as quantised values of a unit normal distribution leave them."""
    codes = PAGE * case["d"]
    words = torch.randint(-2 ** 63, 2 ** 63 - 1, (*shape, codes // 8), device="cuda", generator=dev, dtype=torch.int64)
    pairs = 2 * PAGE * (case["d"] // case["group"])
    u = torch.rand(*shape, pairs, 2, device="cuda", generator=dev)
    params = torch.stack([0.2 + 0.1 * u[..., 0], -2.5 + u[..., 1]], -1).bfloat16()
    return torch.cat([words.view(torch.uint8), params.view(torch.uint8).flatten(-2)], -1)


def _table(lens, pool, width, host):
    pages = -(-lens // PAGE)
    table = np.full((len(lens), width), -1, dtype=np.int64)
    table[np.arange(width) < pages[:, None]] = host.permutation(pool)[:pages.sum()]
    return table


def _prepare_store(case, host, dev):
    seqs, rows, hq, hkv, d = (case[k] for k in ("seqs", "rows", "hq", "hkv", "d"))
    if case["decode"]:
        n = np.ones(seqs, dtype=np.int64)
    else:
        n = np.diff(np.concatenate([[0], np.sort(host.integers(0, rows + 1, seqs - 1)), [rows]]))
    lens = n + host.integers(case["ctx_lo"], case["ctx_hi"] + 1, seqs)
    pool = seqs * (case["ctx_hi"] // PAGE + 2) + rows // PAGE + 1
    width = -(-int(lens.max()) // PAGE)
    qkv = _randn(dev, rows, hq + 2 * hkv, d, dtype=DTYPES[case["dtype"]])       # what a fused projection leaves
    freq = 10000.0 ** -(np.arange(case["rot"] // 2) * 2.0 / max(1, case["rot"]))
    scratch = torch.zeros(pool, 2, PAGE, hkv, d, dtype=torch.bfloat16, device="cuda")
    return dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], pages=_slabs(case, (pool, hkv), dev),
                block_table=_dev(_table(lens, pool, width, host)), seq_lens=_dev(lens),
                cu_q_lens=None if case["decode"] else _dev(np.concatenate([[0], np.cumsum(n)])), inv_freq=_dev(freq, torch.float32),
                scratch=scratch, k_cache=scratch[:, 0], v_cache=scratch[:, 1], to_table=_dev(_table(lens, pool, width, host)))


def _prepare_attend(case, host, dev):
    seqs, hq, hkv, d = (case[k] for k in ("seqs", "hq", "hkv", "d"))
    lens = host.integers(case["lo"], case["hi"] + 1, seqs)
    lens[0] = case["hi"]
    pool = int((-(-lens // PAGE)).sum()) * 9 // 8 + 1
    state = dict(q=_randn(dev, seqs, hq, d), pages=_slabs(case, (pool, hkv), dev), block_table=_dev(_table(lens, pool, -(-case["hi"] // PAGE), host)),
                 seq_lens=_dev(lens), spans=None, head_mask=None, alpha=None, steer_vec=None)
    if case["spans"]:                              # the passages that a sequence is cut into
        cuts = np.sort((host.random((seqs, case["spans"] - 1)) * lens[:, None]).astype(np.int64), axis=1)
        edges = np.concatenate([np.zeros((seqs, 1)), cuts, lens[:, None]], axis=1)
        state["spans"] = _dev(np.stack([edges[:, :-1], edges[:, 1:]], -1))
        state["head_mask"] = torch.zeros(hq, dtype=torch.uint8)
        state["head_mask"][host.permutation(hq)[:case["probed"]].copy()] = 1
    if case["steer"]:
        state["alpha"] = torch.as_tensor(np.where(host.random(hq) < 0.25, 0.8, 0.0)).float()
        state["steer_vec"] = _randn(dev, hq, d, dtype=torch.float32) * 0.1
    return state


def _prepare_copy(case, host, dev):
    order = host.permutation(case["pages"])[:2 * case["pairs"]].reshape(2, -1).T
    order = np.where(host.random((case["pairs"], 1)) < 0.1, -1, order)           # sequences that had nothing to copy
    caches = _slabs(case, (case["layers"], case["pages"], case["hkv"]), dev)
    return dict(caches=caches, layers=list(caches), pairs=_dev(order))


def _prepare_sample(case, host, dev):
    rows, filters = case["rows"], case["filters"]
    state = dict(logits=_randn(dev, rows, case["vocab"], dtype=torch.float32).mul_(3).to(DTYPES[case["dtype"]]),
                 uniform=torch.rand(rows, device="cuda", generator=dev),
                 temperature=_dev(np.where(host.random(rows) < 0.1, 0.0, 0.3 + host.random(rows)), torch.float32), top_k=None, top_p=None, min_p=None)
    if filters in ("all", "top_k"):                # some requests have none
        state["top_k"] = _dev(np.where(host.random(rows) < 0.4, 0, 10 ** (3 * host.random(rows))))
    if filters in ("all", "top_p"):
        state["top_p"] = _dev(np.where(host.random(rows) < 0.3, 1.0, 0.5 + 0.49 * host.random(rows)), torch.float32)
    if filters in ("all", "min_p"):
        state["min_p"] = _dev(np.where(host.random(rows) < 0.5, 0.0, 0.2 * host.random(rows)), torch.float32)
    return state


# ---------------------------------------------------------------------------------- the pages, plainly
def _places(d, values):
    """Byte within its section and shift of the code of every (token, element)."""
    e, t = torch.arange(d, device="cuda"), torch.arange(PAGE, device="cuda")[:, None]
    if not values:
        byte = t * (d // 2) + ((e // 8) % 4 * (d // 32) + e // 32) * 4 + e % 8 // 2
        return byte, (e % 2 * 4).to(torch.uint8).expand(PAGE, d)
    row = (t >> 1 & 3) | (t & 1) << 2 | t & 8
    unit, nibble = e % 8, e % 32 // 8
    if d == 128:
        unit = unit ^ (row & 2) * 2
    return row * (d // 2) + unit * (d // 16) + e // 32 * 2 + nibble // 2, (nibble % 2 * 4).to(torch.uint8).expand(PAGE, d)


def _unpack(slabs, case):
    """Keys and values ``[..., 16, D]`` of slabs ``[..., bytes]``, in 32 bits."""
    d, ng = case["d"], case["d"] // case["group"]
    section, pairs = PAGE * d // 2, PAGE * ng * 4
    params = slabs[..., 2 * section:].contiguous().view(torch.bfloat16).unflatten(-1, (2, PAGE, ng, 2))
    out = []
    for part in (0, 1):
        byte, shift = _places(d, part == 1)
        codes = (slabs[..., (byte + part * section).flatten()].unflatten(-1, (PAGE, d)) >> shift) & 15
        step, lo = (params[..., part, :, :, i].float()[..., None] for i in (0, 1))
        out.append((lo + step * codes.unflatten(-1, (ng, case["group"])).float()).flatten(-2))
    return out


def _quantise(x, case):
    """Codes ``[..., D]``, step and lowest value ``[..., groups]`` of bf16 rows."""
    g = x.float().unflatten(-1, (-1, case["group"]))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    step = ((hi - lo) / 15).bfloat16().float()
    step = torch.where(step < 2.0 ** -100, 0.0, step)
    codes = torch.where(step > 0, ((g - lo).double() / step.double()).round(), 0).clamp(0, 15)   # values next to a border
    return codes.to(torch.uint8).flatten(-2), step[..., 0], lo[..., 0]


# ------------------------------------------------------------------------------------------- one pass
def run(state):
    return {"store": _run_store, "attend": _run_attend, "copy": _run_copy, "sample": _run_sample}[state["case"]["op"]](state)


def _run_store(s):
    case = s["case"]
    if own:
        eng = library()
        q_out = eng.hook_rope_append_q4(q=s["q"], k=s["k"], v=s["v"], pages=s["pages"], block_table=s["block_table"], seq_lens=s["seq_lens"],
                                        cu_q_lens=s["cu_q_lens"], inv_freq=s["inv_freq"])
        eng.hook_cache_read_q4(s["pages"], s["block_table"], s["seq_lens"], k_cache=s["k_cache"], v_cache=s["v_cache"], to_table=s["to_table"])
        return [q_out, s["scratch"]]
    rows = torch.arange(case["rows"], device="cuda")
    lens = s["seq_lens"].long()
    if s["cu_q_lens"] is None:
        seq, at = rows, lens - 1
    else:
        cu = s["cu_q_lens"].long()
        seq = torch.searchsorted(cu, rows, right=True) - 1
        at = lens[seq] - cu[seq + 1] + rows
    angle = at.double()[:, None] * s["inv_freq"].double()
    cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    q_out = _rotate(s["q"].float(), cos, sin, case["rot"]).bfloat16()
    d, ng = case["d"], case["d"] // case["group"]
    section = PAGE * d // 2
    page, slot = s["block_table"].long()[seq, at // PAGE], at % PAGE
    head = torch.arange(case["hkv"], device="cuda")
    flat = s["pages"].view(-1)
    base = (page[:, None] * case["hkv"] + head) * slab_bytes(case)                # where each row's slabs begin
    for part, x in ((0, _rotate(s["k"].float(), cos, sin, case["rot"]).bfloat16()), (1, s["v"].bfloat16())):
        codes, step, lo = _quantise(x, case)
        byte, shift = (p[slot] for p in _places(d, part == 1))                    # [rows, D]
        packed = torch.zeros(case["rows"], case["hkv"], section, dtype=torch.uint8, device="cuda")
        packed.scatter_add_(2, byte[:, None].expand_as(codes), codes << shift[:, None])
        mine = byte.sort(1).values[:, ::2]                                        # a row's bytes, each named by two elements
        flat[base[..., None] + part * section + mine[:, None]] = packed.gather(2, mine[:, None].expand(-1, case["hkv"], -1))
        pair = torch.stack([step, lo], -1).bfloat16().view(torch.uint8).flatten(-2)
        first = base + 2 * section + (part * PAGE + slot[:, None]) * ng * 4
        flat[first[..., None] + torch.arange(ng * 4, device="cuda")] = pair
    # back to bf16: all pages of all sequences
    width = s["block_table"].shape[1]
    live = torch.arange(width * PAGE, device="cuda") < lens[:, None]
    who, t = torch.nonzero(live[:, ::PAGE], as_tuple=True)
    k, v = _unpack(s["pages"][s["block_table"].long()[who, t]], case)             # [pages, Hkv, 16, D]
    here = live.unflatten(1, (width, PAGE))[who, t][:, :, None, None]
    to = s["to_table"].long()[who, t]
    for part, x in ((0, k), (1, v)):
        s["scratch"][to, part] = torch.where(here, x.transpose(1, 2).bfloat16(), s["scratch"][to, part])
    return [q_out, s["scratch"]]


def _rotate(x, cos, sin, rot):
    a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)


def _run_attend(s):
    case = s["case"]
    if own:
        out, mass = library().hook_attn_decode_q4(
            q=s["q"], pages=s["pages"], block_table=s["block_table"], seq_lens=s["seq_lens"], spans=s["spans"], head_mask=s["head_mask"],
            alpha=s["alpha"], steer_vec=s["steer_vec"], max_seq_len=case["hi"])
        return [out] if mass is None else [out, mass]
    seqs, hkv, d = case["seqs"], case["hkv"], case["d"]
    k, v = _unpack(s["pages"][s["block_table"].clamp(min=0).long()], case)        # [seqs, pages, Hkv, 16, D]
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in (k, v))                      # [seqs, Hkv, tokens, D]
    at = torch.arange(k.shape[2], device="cuda")
    live = (at < s["seq_lens"][:, None])[:, None, None]
    x = torch.matmul(s["q"].float().unflatten(1, (hkv, -1)), k.transpose(2, 3)) * d ** -0.5
    x = torch.where(live, x, float("-inf"))
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    out = torch.matmul(p, torch.where(live.transpose(2, 3), v, 0.0)).flatten(1, 2)
    if s["alpha"] is not None:
        out = out + s["alpha"].cuda()[:, None] * s["steer_vec"]
    if s["spans"] is None:
        return [out.bfloat16()]
    inside = (at >= s["spans"][..., :1]) & (at < s["spans"][..., 1:])             # [seqs, spans, tokens]
    mass = torch.matmul(p.flatten(1, 2), inside.float().transpose(1, 2))
    return [out.bfloat16(), mass[:, s["head_mask"].cuda() != 0]]


def _run_copy(s):
    if own:
        library().hook_cache_copy_pages_q4(s["layers"], s["pairs"])
        return s["caches"]
    live = s["pairs"][s["pairs"][:, 0] >= 0].long()
    s["caches"][:, live[:, 1]] = s["caches"][:, live[:, 0]]
    return s["caches"]


def _run_sample(s):
    if own:
        return library().hook_sample_tokens(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    x, index = s["logits"].float().sort(dim=1, descending=True, stable=True)      # ties: the lowest index first
    heat = s["temperature"].double()[:, None]
    greedy = heat == 0
    x = x.double()
    w = torch.exp((x - x[:, :1]) / torch.where(greedy, 1.0, heat))                # 64 bits: a number may fall next to a border
    rank = torch.arange(x.shape[1], device="cuda")
    keep = ~greedy | (rank == 0)
    if s["top_k"] is not None:
        keep &= (rank < s["top_k"][:, None]) | (s["top_k"][:, None] <= 0)
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    if s["top_p"] is not None:
        w = torch.where(keep, w, 0.0)
        before = torch.cumsum(w, 1) - w
        keep &= (before < s["top_p"].double()[:, None] * w.sum(1, keepdim=True)) | (s["top_p"][:, None] >= 1)
    w = torch.zeros_like(w).scatter_(1, index, torch.where(keep, w, 0.0))
    total = torch.cumsum(w, 1)
    token = torch.searchsorted(total, s["uniform"].double()[:, None] * total[:, -1:], right=True)[:, 0]
    last = x.shape[1] - 1 - (w > 0).flip(1).int().argmax(1)
    return torch.minimum(token, last).int()


# ------------------------------------------------------------------------------------------------ work
def work(case):
    if case["op"] == "sample":
        values = case["rows"] * case["vocab"]
        return dict(bytes=values * (4 if case["dtype"] == "fp32" else 2) + case["rows"] * 24, flops=values)
    slab = slab_bytes(case) * case["hkv"]                                         # of one page
    if case["op"] == "copy":
        return dict(bytes=2 * 0.9 * case["pairs"] * case["layers"] * slab, flops=0)
    if case["op"] == "store":
        size = 4 if case["dtype"] == "fp32" else 2
        tokens = case["rows"] + case["seqs"] * (case["ctx_lo"] + case["ctx_hi"]) / 2
        heads = case["hq"] + 2 * case["hkv"]
        return dict(bytes=case["rows"] * (heads * case["d"] * size + case["hq"] * case["d"] * 2) + case["rows"] * slab / PAGE + tokens * slab / PAGE +
                    tokens * 2 * case["hkv"] * case["d"] * 2, flops=case["rows"] * heads * case["rot"] * 3)
    tokens = case["seqs"] * (case["lo"] + case["hi"]) / 2
    return dict(bytes=tokens * slab / PAGE + case["seqs"] * (case["hq"] * case["d"] * 4 + case["spans"] * case["probed"] * 4),
                flops=4 * tokens * case["hq"] * case["d"])


# ---------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    if case["op"] in ("sample", "copy"):
        return None                                # whole numbers
    return {"store": _exact_store, "attend": _exact_attend}[case["op"]](prepare(case, seed), case)


def _element(case):
    """For each section, (byte of the slab, shift) of the code of token t, element e: one element at a time."""
    d, where = case["d"], np.zeros((2, 2, PAGE, case["d"]), dtype=np.int64)
    for t in range(PAGE):
        line = [0, 4, 1, 5, 2, 6, 3, 7][t % 8] + t // 8 * 8                       # even tokens first
        for e in range(d):
            chunk, word = divmod(e, 8)
            where[0, :, t, e] = t * d // 2 + 4 * (chunk % 4 * (d // 32) + chunk // 4) + word // 2, 4 * (word % 2)
            quarter, rest = divmod(e, 32)
            unit = rest % 8 ^ (4 if d == 128 and line % 4 > 1 else 0)
            where[1, :, t, e] = PAGE * d // 2 + line * d // 2 + unit * (d // 16) + 2 * quarter + rest // 16, 4 * (rest // 8 % 2)
    return torch.from_numpy(where).cuda()


def _slab_values(slab, case, where):
    """Keys and values in 64 bits of some pages ``[n, Hkv, bytes]`` as ``[n * 16, Hkv, D]``."""
    d, per = case["d"], case["group"]
    params = slab[..., PAGE * d:].contiguous().view(torch.bfloat16).double().view(*slab.shape[:2], 2, PAGE, d // per, 2)
    got = []
    for part in (0, 1):
        byte, shift = where[part]
        code = (slab[:, :, byte.reshape(-1)].long().view(*slab.shape[:2], PAGE, d) >> shift) % 16
        step = params[:, :, part, :, :, 0].repeat_interleave(per, -1)
        low = params[:, :, part, :, :, 1].repeat_interleave(per, -1)
        got.append((code * step + low).permute(0, 2, 1, 3).reshape(-1, slab.shape[1], d))
    return got


def _exact_store(s, case):
    """Sequence by sequence: what its pages stand for, with the new rows' codes in their place."""
    d, rot, where = case["d"], case["rot"], _element(case)
    lens = s["seq_lens"].tolist()
    cu = s["cu_q_lens"].tolist() if s["cu_q_lens"] is not None else list(range(len(lens) + 1))
    q_out = s["q"].double()
    scratch = s["scratch"].double()
    turn = lambda at: torch.polar(torch.ones(len(at), rot // 2, dtype=torch.float64, device="cuda"), at[:, None] * s["inv_freq"].double())[:, None]  # noqa: E731

    def turned(x, z):
        y = x.double()
        c = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * z
        y[..., :rot // 2], y[..., rot // 2:rot] = c.real, c.imag
        return y

    def stored(x):
        y = x.to(torch.bfloat16).float().unflatten(2, (d // case["group"], case["group"]))
        low = y.min(3, keepdim=True)[0]
        step = ((y.max(3, keepdim=True)[0] - low) / 15).to(torch.bfloat16).double()
        code = torch.round((y - low).double() / step.clamp(min=1e-300)).clamp(max=15)
        return (code * step + low.double()).flatten(2)

    for i, L in enumerate(lens):
        n, r = cu[i + 1] - cu[i], slice(cu[i], cu[i + 1])
        at = torch.arange(L - n, L, device="cuda", dtype=torch.float64)
        z = turn(at)
        k, v = _slab_values(s["pages"][s["block_table"][i, :-(-L // PAGE)].long()], case, where)
        if n:
            q_out[r] = turned(s["q"][r], z)
            k[L - n:L], v[L - n:L] = stored(turned(s["k"][r], z)), stored(s["v"][r].to(torch.bfloat16))
        for j in range(-(-L // PAGE)):
            to, last = s["to_table"][i, j], min(PAGE, L - j * PAGE)
            scratch[to, 0, :last], scratch[to, 1, :last] = k[j * PAGE:j * PAGE + last], v[j * PAGE:j * PAGE + last]
    return [q_out, scratch]


def _exact_attend(s, case):
    """Sequence by sequence, head by head."""
    where = _element(case)
    per = case["hq"] // case["hkv"]
    probed = [] if s["head_mask"] is None else torch.nonzero(s["head_mask"])[:, 0].tolist()
    out = torch.empty(case["seqs"], case["hq"], case["d"], dtype=torch.float64, device="cuda")
    mass = torch.empty(case["seqs"], len(probed), case["spans"], dtype=torch.float64, device="cuda")
    for i, L in enumerate(s["seq_lens"].tolist()):
        k, v = _slab_values(s["pages"][s["block_table"][i, :-(-L // PAGE)].long()], case, where)
        spans = [] if s["spans"] is None else s["spans"][i].tolist()
        for h in range(case["hq"]):
            p = torch.softmax(k[:L, h // per] @ s["q"][i, h].double() / case["d"] ** 0.5, 0)
            out[i, h] = p @ v[:L, h // per]
            if s["alpha"] is not None:
                out[i, h] += s["alpha"][h].double() * s["steer_vec"][h].double()
            if h in probed:
                for j, (a, b) in enumerate(spans):
                    mass[i, probed.index(h), j] = p[a:b].sum()
    return [out, mass] if probed else [out]
