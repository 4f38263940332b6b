"""Operators for serving many sequences from one pool of pages: what they compute, and the work users give them.

Three kinds of call, each over the range its users meet:

* ``append``     sdsat_paged_append: a call's new tokens, a ragged chunk of each sequence, leave a linear layer as rows
                 q | k | v; queries and keys are normalised by head and rotated, keys and values go to the sequences'
                 pages, queries to the attention;
* ``attention``  sdsat_paged_attention: each new token's queries against its sequence's pages, for chunks of prompts,
                 draft and verify blocks (tree masks) and single tokens, in one call;
* ``adjust``     sdsat_adjust_logits: logits rows on their way to verification: penalties for tokens that the row's
                 context holds (the drafts ahead of it among them), biases, and ids that a grammar does not allow.

``run`` computes each either from elementary torch operations (``own`` false) or through the library.  Heads of the
7B, 13B and tiny decoders and layouts whose query heads share key heads; pages lie scattered over the pool.
"""
import math

import torch

own = False

PAGE = 32   # slots of a page


def listed():
    return [
        # the draft block (k = 5) of the tiny fp32 decoder: launches and latency
        {"name": "append_tiny", "kind": "append", "dtype": "fp32", "x": "fp32", "heads": 4, "kv": 4, "dh": 64,
         "batch": 1, "n": 6, "ctx": 90, "spare": 0, "layout": "half", "rot": 64, "scaling": "none", "far": 0,
         "norm": False},
        # draft blocks of eight sequences at 7B heads, straight from the library's linear layer (float rows)
        {"name": "append_block_7b", "kind": "append", "dtype": "bf16", "x": "fp32", "heads": 32, "kv": 32, "dh": 128,
         "batch": 8, "n": 6, "ctx": 1013, "spare": 0, "layout": "half", "rot": 128, "scaling": "none", "far": 0,
         "norm": False},
        # one token each for 64 long sequences, eight key heads, norms by head, frequencies scaled by parts
        {"name": "append_decode_64", "kind": "append", "dtype": "bf16", "x": "bf16", "heads": 32, "kv": 8, "dh": 128,
         "batch": 64, "n": 1, "ctx": 1990, "spare": 0, "layout": "half", "rot": 128, "scaling": "parts",
         "far": 100000, "norm": True},
        # prompts of about 2000 tokens behind a cached instruction, half of each head rotated as neighbouring pairs
        {"name": "append_prefill", "kind": "append", "dtype": "bf16", "x": "bf16", "heads": 32, "kv": 8, "dh": 128,
         "batch": 4, "n": 2047, "ctx": 500, "spare": 9, "layout": "interleaved", "rot": 64, "scaling": "none",
         "far": 0, "norm": True},
        # the draft block of the tiny fp32 decoder
        {"name": "attn_tiny", "kind": "attention", "dtype": "fp32", "heads": 4, "kv": 4, "dh": 64, "batch": 1, "n": 6,
         "ctx": 90, "chunk": 0, "chunk_ctx": 0, "tree": 0, "window": 0, "spare": 0},
        # draft trees (k = 5, width 2) of four sequences at 7B heads
        {"name": "attn_tree_7b", "kind": "attention", "dtype": "bf16", "heads": 32, "kv": 32, "dh": 128, "batch": 4,
         "n": 11, "ctx": 1500, "chunk": 0, "chunk_ctx": 0, "tree": 2, "window": 0, "spare": 0},
        # one token each for 64 ragged sequences
        {"name": "attn_decode_64", "kind": "attention", "dtype": "bf16", "heads": 32, "kv": 8, "dh": 128, "batch": 64,
         "n": 1, "ctx": 4000, "chunk": 0, "chunk_ctx": 0, "tree": 0, "window": 0, "spare": 0},
        # one token of a single, very long sequence
        {"name": "attn_decode_long", "kind": "attention", "dtype": "bf16", "heads": 32, "kv": 8, "dh": 128, "batch": 1,
         "n": 1, "ctx": 130000, "chunk": 0, "chunk_ctx": 0, "tree": 0, "window": 0, "spare": 0},
        # a server's step: a piece of a long prompt beside the single tokens of 31 sequences
        {"name": "attn_mixed", "kind": "attention", "dtype": "bf16", "heads": 32, "kv": 8, "dh": 128, "batch": 31,
         "n": 1, "ctx": 2500, "chunk": 1001, "chunk_ctx": 5000, "tree": 0, "window": 0, "spare": 4},
        # the second half of an 8192-token prompt
        {"name": "attn_prefill", "kind": "attention", "dtype": "bf16", "heads": 32, "kv": 8, "dh": 128, "batch": 1,
         "n": 4096, "ctx": 4096, "chunk": 0, "chunk_ctx": 0, "tree": 0, "window": 0, "spare": 0},
        # the verify block of a batch-1 loop (k = 5) with penalties over an 800-token history
        {"name": "adjust_b1", "kind": "adjust", "batch": 1, "q": 6, "vocab": 32016, "hist": 800, "bias": "none",
         "grammar": False, "tree": 0},
        # verify blocks of 16 sequences over a large vocabulary: penalties, one bias row for all, a grammar by row
        {"name": "adjust_128k", "kind": "adjust", "batch": 16, "q": 6, "vocab": 128256, "hist": 4000, "bias": "shared",
         "grammar": True, "tree": 0},
    ]


HEADS = [(32, 8, 128, "bf16"), (32, 8, 128, "bf16"), (32, 32, 128, "bf16"), (40, 40, 128, "bf16"), (40, 8, 128, "bf16"),
         (28, 4, 128, "bf16"), (8, 1, 64, "bf16"), (8, 8, 64, "bf16"), (4, 4, 64, "fp32"), (6, 2, 128, "fp32")]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "attention", "attention", "attention", "adjust", "adjust"])
    if kind == "adjust":
        vocab = rng.choice([1000, 1024, 32000, 32016, 32017, 50257, 128256])
        rows = _log_int(rng, 1, min(400, 12_000_000 // vocab))
        batch = rng.choice([b for b in (1, 1, 2, 3, 4, 8, 16, 24) if b <= rows])
        q = min(rows // batch, 64)
        return {"kind": "adjust", "batch": batch, "q": q, "vocab": vocab, "hist": _log_int(rng, 1, 16000),
                "bias": rng.choice(["none", "shared", "each"]), "grammar": rng.random() < 0.6,
                "tree": 2 if q >= 3 and q % 2 == 1 and rng.random() < 0.5 else 0}
    heads, kv, dh, dtype = rng.choice(HEADS)
    if kind == "append":
        n = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 17, 4000)])
        batch = _log_int(rng, 1, min(100, max(1, 8000 // n)))
        return {"kind": "append", "dtype": dtype, "x": "fp32" if dtype == "fp32" else rng.choice(["fp32", "bf16"]),
                "heads": heads, "kv": kv, "dh": dh, "batch": batch, "n": n, "ctx": rng.choice([0, _log_int(rng, 1, 4000)]),
                "spare": rng.choice([0, 0, 5]), "layout": rng.choice(["half", "interleaved"]),
                "rot": rng.choice([dh, dh, dh // 2, 24]), "scaling": rng.choice(["none", "linear", "ntk", "parts"]),
                "far": rng.choice([0, 0, 100000, 1000000]), "norm": rng.random() < 0.5}
    case = {"kind": "attention", "dtype": dtype, "heads": heads, "kv": kv, "dh": dh, "chunk": 0, "chunk_ctx": 0,
            "tree": 0, "window": rng.choice([0, 0, 0, _log_int(rng, 1, 2000)]), "spare": rng.choice([0, 0, 7])}
    most = 2_000_000 if dtype == "bf16" else 400_000   # scores of a head
    if rng.random() < 0.4:   # chunks of prompts
        n = _log_int(rng, 20, 2500)
        ctx = rng.choice([0, _log_int(rng, 1, 6000)])
        batch = rng.randint(1, max(1, min(6, 4 * most // (n * (n + ctx)))))
        return dict(case, batch=batch, n=n, ctx=ctx)
    n = rng.choice([1, 1, rng.randint(2, 16)])
    batch = _log_int(rng, 1, 64)
    ctx = _log_int(rng, 1, min(130000, 3_000_000 // (batch * max(kv, 8))))
    if n >= 3 and n % 2 == 1 and rng.random() < 0.7:
        return dict(case, batch=batch, n=n, ctx=ctx, tree=2, window=0)
    if rng.random() < 0.3:   # a piece of a prompt among them
        case["chunk"] = _log_int(rng, 17, 1000)
        case["chunk_ctx"] = rng.choice([0, _log_int(rng, 1, 2000)])
    return dict(case, batch=batch, n=n, ctx=ctx)


# ------------------------------------------------------------------ inputs (from the seed alone)
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _randn(shape, dtype, g):
    """N(0, 1), at most 2^28 values at a time in float32."""
    if dtype == torch.float32:
        return torch.randn(shape, generator=g, device="cuda")
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    for lo in range(0, flat.numel(), 1 << 28):
        part = flat[lo:lo + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda"))
    return t


def _sequences(case):
    """(new tokens, cached tokens) of every sequence, ragged."""
    n, ctx = case["n"], case["ctx"]
    seqs = [(n - 7 * b % n if n > 16 else n, max(0, ctx - 19 * b)) for b in range(case["batch"])]
    if case.get("chunk"):
        seqs.insert(0, (case["chunk"], case["chunk_ctx"]))
    return seqs


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _plan(case, g):
    """Chunk borders, cached lengths and page tables (pages scattered over the pool; -1 where a sequence has none, or,
    for appending and ahead of a window, needs none)."""
    seqs = _sequences(case)
    start = [0]
    for n, _ in seqs:
        start.append(start[-1] + n)
    width = max(-(-(n + ctx) // PAGE) for n, ctx in seqs)
    first = []
    for n, ctx in seqs:
        lo = ctx if case["kind"] == "append" else ctx - case["window"] + 1 if case["window"] else 0
        first.append(max(0, lo) // PAGE)
    counts = [-(-(n + ctx) // PAGE) - f for (n, ctx), f in zip(seqs, first)]
    n_pages = sum(counts) + 3
    ids = torch.randperm(n_pages, generator=g, device="cuda").int()
    pages = torch.full((len(seqs), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, (f, c) in enumerate(zip(first, counts)):
        pages[b, f:f + c] = ids[at:at + c]
        at += c
    return {"start": _ints(start), "len": _ints([ctx for _, ctx in seqs]), "pages": pages, "n_pages": n_pages,
            "unused": ids[at].long(), "rows": start[-1] + case["spare"], "max_q": max(n for n, _ in seqs),
            "max_len": max(n + ctx for n, ctx in seqs)}


def _pool(case, plan, g):
    """K [pages, key heads, slots, head_dim] and V [pages, key heads, head_dim, places]: the slot 16a + 4g + r of a page
    at place 8g + 4a + r."""
    k = _randn((plan["n_pages"], case["kv"], PAGE, case["dh"]), _dtype(case["dtype"]), g)
    return k, _randn((plan["n_pages"], case["kv"], case["dh"], PAGE), _dtype(case["dtype"]), g)


def _tree_mask(q, width):
    """Ancestor masks of a draft tree: root, the chain, then the other candidates of each depth as leaves."""
    k = (q - 1) // width
    mask = [1] + [(1 << (j + 1)) - 1 for j in range(1, k + 1)]
    for j in range(1, k + 1):
        for _ in range(width - 1):
            mask.append(((1 << j) - 1) | (1 << len(mask)))
    return mask


def _append_inputs(case, plan, g):
    """Rows q | k | v, positions (those of the slots, moved by `far`) and the norms' gains."""
    rows, dh = plan["rows"], case["dh"]
    x = _randn((rows, (case["heads"] + 2 * case["kv"]) * dh), _dtype(case["x"]), g)
    pos = torch.zeros(rows, dtype=torch.int32)
    at = 0
    for n, ctx in _sequences(case):
        pos[at:at + n] = torch.arange(ctx, ctx + n) + case["far"]
        at += n
    gains = 1 + 0.1 * torch.randn((2, dh), generator=g, device="cuda") if case["norm"] else None
    return x, pos.cuda(), gains


def _logit_inputs(case, g):
    """Logits, histories (with ids that are not in the vocabulary), the block's tokens and masks, penalties by sequence,
    biases, allowed ids (a bit each)."""
    batch, q, vocab, dev = case["batch"], case["q"], case["vocab"], "cuda"
    s = {"logits": torch.randn((batch * q, vocab), generator=g, device=dev).mul_(4.0)}
    lens = [max(1, case["hist"] - 37 * b) for b in range(batch)]
    words = 1 + vocab // 20   # text repeats itself
    s["history"] = torch.randint(0, words, (batch, case["hist"]), generator=g, device=dev).int()
    s["history"][:, ::50] = vocab
    s["hist_len"], s["prompt_len"] = _ints(lens), _ints([n // 2 for n in lens])
    s["tokens"] = torch.randint(0, words, (batch, q), generator=g, device=dev).int()
    mask = _tree_mask(q, case["tree"]) if case["tree"] else None
    s["mask"] = torch.tensor(mask * batch, dtype=torch.int64, device=dev) if mask else None
    kinds = torch.tensor([[1.2, 0.0, 0.0], [1.0, 0.5, 0.3], [1.1, 0.1, 0.0], [0.9, -0.2, 0.4]])
    s["penalties"] = kinds[torch.arange(batch) % 4].t().contiguous().to(dev)   # repetition, frequency, presence
    s["bias"] = None
    if case["bias"] != "none":
        shape = (1 if case["bias"] == "shared" else batch, vocab)
        s["bias"] = torch.randn(shape, generator=g, device=dev)
        s["bias"][:, ::97] = -math.inf
    s["allowed"] = None
    if case["grammar"]:
        s["allowed"] = torch.randint(-2**31, 2**31, (batch * q, -(-vocab // 32)), generator=g, device=dev).int()
    return s


# ------------------------------------------------------------------ rotary frequencies
BASE, CTX, FACTOR, LOW, HIGH = 1e6, 16384.0, 8.0, 1.0, 4.0
EPS = 1e-5


def _mscale(case):
    return 0.1 * math.log(FACTOR) + 1 if case["scaling"] == "parts" else 1.0


def _frequencies(case):
    """Angle per position of each pair, as scaled for long contexts."""
    r = case["rot"]
    j = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    base = BASE * FACTOR ** (r / (r - 2)) if case["scaling"] == "ntk" else BASE
    f = base ** (-2 * j / r)
    if case["scaling"] == "linear":
        return f / FACTOR
    if case["scaling"] == "parts":   # slow pairs as for a longer context, fast ones as they are
        keep = ((CTX * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        return f / FACTOR * (1 - keep) + f * keep
    return f


# ------------------------------------------------------------------ what a program holds before the call
def prepare(case, seed):
    """Inputs, alike for both forms; for the library's calls also its handle and its descriptions of the call."""
    g = _gen(seed)
    if case["kind"] == "adjust":
        s = _logit_inputs(case, g)
        s["case"], s["out"] = case, torch.empty_like(s["logits"])
        if own:
            s["ctx"] = _context(case)
            from paper_2403_18647_amd import binding as B
            s["rules"] = B.logit_rules(history=s["history"], history_len=s["hist_len"], prompt_len=s["prompt_len"],
                                       tokens=s["tokens"], mask=s["mask"], penalties=s["penalties"], bias=s["bias"],
                                       allowed=s["allowed"])
        return s
    s = _plan(case, g)
    s["case"] = case
    s["k"], s["v"] = _pool(case, s, g)
    if case["kind"] == "append":
        s["x"], s["pos"], s["gains"] = _append_inputs(case, s, g)
        s["out"] = torch.zeros((s["rows"], case["heads"] * case["dh"]), dtype=s["k"].dtype, device="cuda")
    else:
        s["q"] = 2 * _randn((s["rows"], case["heads"] * case["dh"]), s["k"].dtype, g)
        s["out"] = torch.zeros_like(s["q"])
        s["mask"] = None
        if case["tree"]:
            s["mask"] = torch.tensor(_tree_mask(case["n"], case["tree"]) * case["batch"] + [0] * case["spare"],
                                     dtype=torch.int64, device="cuda")
    if own:
        from paper_2403_18647_amd import binding as B
        s["paged"] = B.Paged(B.sdsat_paged_config(
            n_heads=case["heads"], n_kv_heads=case["kv"], head_dim=case["dh"],
            dtype=B.DTYPE_BF16 if case["dtype"] == "bf16" else B.DTYPE_FP32, n_pages=s["n_pages"], max_rows=s["rows"],
            max_batch=len(s["len"]), max_ctx=s["max_len"]))
        s["batch"] = B.paged_batch(s["start"], s["len"], s["pages"], s["rows"], s["max_q"], s["max_len"])
        if case["kind"] == "append":
            s["rope"] = B.sdsat_rope_init(layout=case["layout"], rot_dims=case["rot"], base=BASE,
                                          scaling=case["scaling"], factor=FACTOR, ctx=CTX, low=LOW, high=HIGH,
                                          mscale=_mscale(case))
    return s


def _context(case):
    """A library context of this vocabulary (the calls here read no weights)."""
    from paper_2403_18647_amd import binding as B
    from paper_2403_18647_amd import synth
    sh = synth.small_shape(n_layers=1, d_ffn=64, vocab=case["vocab"], n_adaptive=0)
    w = [torch.zeros(synth.tensor_shape(sh, n), device="cuda") for n in synth.tensor_names(sh)]
    return B.Context(B.make_config(sh, case["batch"], 32, case["q"]), w)


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "append":
        return _plain_append(s, case)
    if case["kind"] == "attention":
        return _plain_attention(s, case)
    return _plain_adjust(s, case)


def _run_own(s, case):
    from paper_2403_18647_amd import binding as B
    if case["kind"] == "append":
        q_gain, k_gain = s["gains"] if s["gains"] is not None else (None, None)
        B.sdsat_paged_append(s["paged"].handle, s["batch"], s["k"], s["v"], s["x"], s["rope"], s["pos"], q_gain, k_gain,
                             EPS, s["out"])
        return s["out"], s["k"], s["v"]
    if case["kind"] == "attention":
        B.sdsat_paged_attention(s["paged"].handle, s["batch"], s["k"], s["v"], s["q"], s["mask"], case["window"], 0.0,
                                s["out"])
        return s["out"]
    B.sdsat_adjust_logits(s["ctx"].handle, case["batch"], case["q"], s["logits"], s["rules"], s["out"])
    return s["out"]


def _owner(s):
    """The sequence of each row (of the rows behind the last one: past the end), and its slot."""
    row = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(s["start"], row, right=True, out_int32=True) - 1
    at = b.clamp(max=len(s["len"]) - 1).long()
    return b < len(s["len"]), at, row - s["start"][at] + s["len"][at]


def _plain_append(s, case):
    heads, kv, dh, r = case["heads"], case["kv"], case["dh"], case["rot"]
    x = s["x"].float().view(s["rows"], heads + 2 * kv, dh)
    qk, v = x[:, :heads + kv], x[:, heads + kv:]
    if s["gains"] is not None:
        gain = s["gains"].repeat_interleave(torch.tensor([heads, kv], device="cuda"), 0, output_size=heads + kv)
        qk = qk * torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS) * gain
    angle = s["pos"].double()[:, None] * _frequencies(case)
    cos, sin = (torch.cos(angle) * _mscale(case)).float()[:, None], (torch.sin(angle) * _mscale(case)).float()[:, None]
    rest = qk[..., r:]
    if case["layout"] == "half":
        a, c = qk[..., :r // 2], qk[..., r // 2:r]
        qk = torch.cat([a * cos - c * sin, c * cos + a * sin, rest], -1)
    else:
        a, c = qk[..., 0:r:2], qk[..., 1:r:2]
        qk = torch.cat([torch.stack([a * cos - c * sin, c * cos + a * sin], -1).flatten(-2), rest], -1)
    mine, b, slot = _owner(s)
    page = s["pages"][b, (slot // PAGE).clamp(max=s["pages"].shape[1] - 1)].long()
    at = slot % PAGE
    place = at // 4 % 4 * 8 + at // 16 * 4 + at % 4
    # rows behind the last sequence write what a page of no sequence holds
    page, at, place = (torch.where(mine, t, d) for t, d in ((page, s["unused"]), (at, 0), (place, 0)))
    keep = mine[:, None, None]
    s["k"][page, :, at] = torch.where(keep, qk[:, heads:].to(s["k"].dtype), s["k"][page, :, at])
    s["v"][page, :, :, place] = torch.where(keep, v.to(s["v"].dtype), s["v"][page, :, :, place])
    s["out"].copy_(torch.where(mine[:, None], qk[:, :heads].reshape(s["rows"], -1).to(s["out"].dtype), s["out"]))
    return s["out"], s["k"], s["v"]


def _plain_attention(s, case):
    """Sequences of like chunks padded to their longest; the padding goes to a row that is dropped."""
    out = torch.zeros((s["rows"] + 1, s["q"].shape[1]), dtype=s["q"].dtype, device="cuda")
    first = 1 if case["chunk"] else 0
    groups = ([(0, 1, case["chunk"], case["chunk_ctx"])] if first else []) + \
        [(first, len(s["len"]), case["n"], case["ctx"])]
    for lo, hi, n, ctx in groups:
        _plain_group(s, case, lo, hi, n, n + ctx, out)
    return out[:-1]


def _plain_group(s, case, lo, hi, n, width, out):
    kv, dh, dev = case["kv"], case["dh"], "cuda"
    per = case["heads"] // kv
    width = -(-width // PAGE)
    pages = s["pages"][lo:hi, :width].clamp(min=0).long()
    count = hi - lo
    k = s["k"][pages].transpose(1, 2).reshape(count, kv, width * PAGE, dh).float()
    v = s["v"][pages].view(count, width, kv, dh, 4, 2, 4).permute(0, 2, 1, 5, 4, 6, 3).reshape(k.shape).float()
    length = s["len"][lo:hi, None]
    i = torch.arange(n, device=dev)
    row = s["start"][lo:hi, None] + i
    mine = row < s["start"][lo + 1:hi + 1, None]
    held = torch.where(mine, row, 0).long()
    q = s["q"][held].float().view(count, n, kv, per, dh).permute(0, 2, 3, 1, 4).reshape(count, kv, per * n, dh)
    score = torch.matmul(q * (1 / math.sqrt(dh)), k.transpose(2, 3).contiguous())
    slot = torch.arange(width * PAGE, device=dev)
    at = (length + i)[..., None]
    if s["mask"] is None:
        see = slot <= at
        if case["window"]:
            see = see & (slot > at - case["window"])
    else:
        ahead = (slot - length).clamp(0, 63)[:, None]
        see = (slot < length)[:, None] | ((s["mask"][held][..., None] >> ahead & 1 == 1) & (slot < length + n)[:, None])
    score = score.view(count, kv, per, n, -1).masked_fill(~see[:, None, None], -math.inf)
    e = torch.exp(score - score.amax(-1, keepdim=True))
    den = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(count, kv, per * n, -1), v).view(count, kv, per, n, dh) / den
    out[torch.where(mine, row, s["rows"]).long()] = o.permute(0, 3, 1, 2, 4).reshape(count, n, -1).to(out.dtype)


def _plain_adjust(s, case):
    batch, q, vocab = case["batch"], case["q"], case["vocab"]
    z = s["logits"].view(batch, q, vocab)
    i = torch.arange(case["hist"], device="cuda")
    word = s["history"].long()
    known = (i < s["hist_len"][:, None]) & (word >= 0) & (word < vocab)
    word = word.clamp(0, vocab - 1)
    told = known & (i >= s["prompt_len"][:, None])
    zero = torch.zeros((batch, vocab), dtype=torch.int32, device="cuda")
    asked = zero.scatter_add(1, word, (known & ~told).int())
    count = zero.scatter_add(1, word, told.int())[:, None].expand(batch, q, vocab).contiguous()
    j = torch.arange(q, device="cuda")
    see = (j <= j[:, None]).expand(batch, q, q)
    if s["mask"] is not None:
        see = (s["mask"].view(batch, q, 1) >> j & 1) == 1
    block = s["tokens"].long()[:, None].expand(batch, q, q)
    count.scatter_add_(2, block, see.int())
    rep, freq, pres = (t[:, None, None] for t in s["penalties"])
    seen = (count > 0) | (asked > 0)[:, None]
    z = torch.where(seen, torch.where(z > 0, z / rep, z * rep), z)
    z = z - freq * count - pres * (count > 0)
    if s["bias"] is not None:
        z = z + s["bias"][:, None]
    z = z.view(batch * q, vocab)
    if s["allowed"] is not None:
        ids = torch.arange(vocab, device="cuda")
        z = torch.where((s["allowed"][:, ids // 32] >> (ids % 32) & 1) == 1, z, -math.inf)
    return z


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "adjust":
        rows, vocab, batch = case["batch"] * case["q"], case["vocab"], case["batch"]
        by = rows * vocab * 8 + sum(max(1, case["hist"] - 37 * b) for b in range(batch)) * 4
        by += {"none": 0, "shared": vocab * 4, "each": batch * vocab * 4}[case["bias"]]
        by += rows * -(-vocab // 32) * 4 if case["grammar"] else 0
        return {"bytes": by, "flops": 2.0 * rows * vocab}
    seqs = _sequences(case)
    rows = sum(n for n, _ in seqs)
    d, dk, e = case["heads"] * case["dh"], case["kv"] * case["dh"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "append":
        x = 2 if case["x"] == "bf16" else 4
        return {"bytes": rows * (d + 2 * dk) * (x + e) + 4 * rows, "flops": rows * (d + dk) * (7.0 if case["norm"] else 3.0)}
    by, fl, window = 2.0 * rows * d * e, 0.0, case["window"]
    for n, ctx in seqs:
        by += 2 * dk * e * (n + min(ctx, window - 1) if window else n + ctx)
        if window:   # the row at slot s sees min(s + 1, window) slots
            full = max(0, min(n, ctx + n - window + 1))   # rows that see a whole window
            rest = n - full
            seen = full * window + rest * ctx + rest * (rest + 1) / 2
        else:
            seen = n * ctx + n * (n + 1) / 2
        fl += 4.0 * d * seen
    return {"bytes": by, "flops": fl}


# ------------------------------------------------------------------ the same from the definitions in 64 bits
def exact(case, seed):
    g = _gen(seed)
    if case["kind"] == "adjust":
        return _exact_adjust(case, _logit_inputs(case, g))
    plan = _plan(case, g)
    k, v = (t.double() for t in _pool(case, plan, g))
    if case["kind"] == "append":
        return _exact_append(case, plan, k, v, *_append_inputs(case, plan, g))
    return _exact_attention(case, plan, k, v, 2 * _randn((plan["rows"], case["heads"] * case["dh"]),
                                                         _dtype(case["dtype"]), g))


def _exact_append(case, plan, k, v, x, pos, gains):
    heads, kv, dh, r = case["heads"], case["kv"], case["dh"], case["rot"]
    freq = []
    for j in range(r // 2):
        f = math.exp(-2 * j / r * math.log(BASE))
        if case["scaling"] == "linear":
            f /= FACTOR
        elif case["scaling"] == "ntk":
            f = math.exp(-2 * j / r * (math.log(BASE) + r / (r - 2) * math.log(FACTOR)))
        elif case["scaling"] == "parts":
            turns = CTX / (2 * math.pi / f)
            f = f if turns > HIGH else f / FACTOR if turns < LOW else \
                f * (1 / FACTOR + (1 - 1 / FACTOR) * (turns - LOW) / (HIGH - LOW))
        freq.append(f)
    turn = torch.polar(torch.tensor(_mscale(case), dtype=torch.float64, device="cuda"),
                       pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device="cuda"))
    x = x.double().view(-1, heads + 2 * kv, dh)
    out = torch.zeros((x.shape[0], heads, dh), dtype=torch.float64, device="cuda")
    new = [x[:, :heads].clone(), x[:, heads:heads + kv].clone()]
    for i, t in enumerate(new):
        if gains is not None:
            t /= (t.square().sum(-1, keepdim=True) / dh + EPS).sqrt()
            t *= gains[i].double()
        lo, hi = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2), slice(1, r, 2))
        z = torch.complex(t[..., lo], t[..., hi]) * turn[:, None]
        t[..., lo], t[..., hi] = z.real, z.imag
    v = v.view(-1, kv, dh, 4, 2, 4)
    at = 0
    for b, (n, ctx) in enumerate(_sequences(case)):
        out[at:at + n] = new[0][at:at + n]
        slot = torch.arange(ctx, ctx + n, device="cuda")
        page = plan["pages"][b].long()[slot // PAGE]
        k[page, :, slot % PAGE] = new[1][at:at + n]
        v[page, :, :, slot % 16 // 4, slot % PAGE // 16, slot % 4] = x[at:at + n, heads + kv:]
        at += n
    return out.view(x.shape[0], -1), k, v.view(-1, kv, dh, PAGE)


def _exact_attention(case, plan, k, v, q):
    """One sequence and key head at a time, at most 1024 rows of it."""
    kv, dh = case["kv"], case["dh"]
    per = case["heads"] // kv
    q = q.double().view(-1, kv, per, dh)
    out = torch.zeros_like(q)
    tree = _tree_mask(case["n"], case["tree"]) if case["tree"] else None
    at = 0
    for b, (n, ctx) in enumerate(_sequences(case)):
        first = max(0, ctx - case["window"] + 1) // PAGE if case["window"] else 0
        page = plan["pages"][b, first:-(-(n + ctx) // PAGE)].long()
        slot = torch.arange(first * PAGE, n + ctx, device="cuda")
        for lo in range(0, n, 1024):
            i = torch.arange(lo, min(n, lo + 1024), device="cuda")
            hidden = slot > (ctx + i)[:, None]
            if case["window"]:
                hidden |= slot <= (ctx + i)[:, None] - case["window"]
            if tree:
                rows = torch.tensor([[not m >> j & 1 for j in range(n)] for m in tree], device="cuda")
                hidden = torch.cat([torch.zeros((n, ctx), dtype=torch.bool, device="cuda"), rows], 1)
            for h in range(kv):
                kk = k[page, h].view(-1, dh)[:len(slot)]
                vv = v[page, h].view(-1, dh, 4, 2, 4).permute(0, 3, 2, 4, 1).reshape(-1, dh)[:len(slot)]
                sc = torch.matmul(q[at + i, h].transpose(0, 1).reshape(-1, dh), kk.t().contiguous()) / math.sqrt(dh)
                w = sc.view(per, len(i), -1).masked_fill(hidden, -math.inf).softmax(-1)
                out[at + i, h] = torch.matmul(w.view(per * len(i), -1), vv).view(per, len(i), dh).transpose(0, 1)
        at += n
    return out.view(len(q), -1)


def _exact_adjust(case, s):
    batch, q, vocab = case["batch"], case["q"], case["vocab"]
    z = s["logits"].double().view(batch, q, vocab)
    tree = _tree_mask(q, case["tree"]) if case["tree"] else [(2 << j) - 1 for j in range(q)]
    pen = s["penalties"].double()
    for b in range(batch):
        hist = s["history"][b, :int(s["hist_len"][b])].long()
        prompt = int(s["prompt_len"][b])
        old, said = (torch.bincount(t[t < vocab], minlength=vocab) for t in (hist[:prompt], hist[prompt:]))
        for j in range(q):
            ahead = torch.tensor([i for i in range(q) if tree[j] >> i & 1], device="cuda")
            c = said + torch.bincount(s["tokens"][b].long()[ahead], minlength=vocab)
            row = z[b, j]
            factor = torch.where(row > 0, 1 / pen[0, b], pen[0, b])
            row *= torch.where(old + c > 0, factor, torch.ones_like(factor))
            row -= pen[1, b] * c + pen[2, b] * (c > 0)
            if s["bias"] is not None:
                row += s["bias"][b if case["bias"] == "each" else 0].double()
            if s["allowed"] is not None:
                bits = s["allowed"][b * q + j][:, None] >> torch.arange(32, device="cuda") & 1
                row[bits.flatten()[:vocab] == 0] = -math.inf
    return z.view(batch * q, vocab)
