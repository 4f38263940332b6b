"""Operators for sampling and ranking several completions of one prompt: what they compute, and the work users give them.

Three kinds of call, each over the range its users meet:

* ``reorder``    sdsat_kv_reorder: sequences of a batch continue from other sequences' caches (a prompt forked into
                 samples, beams that follow their parents, survivors moved into the rows of finished sequences);
* ``attention``  sdsat_attention_shared: block attention of sequences that share a long prefix, held by the first of
                 each group, and have their own slots behind it;
* ``logprobs``   sdsat_token_logprobs: the log probabilities of given tokens under logits rows, each row's entropy and
                 its most probable alternatives.

``run`` computes each either from elementary torch operations in float32 (``own`` false) or through the library.
Heads, vocabularies and slot counts are those of the 7B, 13B and tiny decoders.  Cached K and V and queries are
N(0, 1), logits N(0, 4) with the last ids of some rows banned (-inf).
"""
import math

import torch

own = False

PAGE = 32   # cache slots that move together


def listed():
    return [
        # a prompt of the tiny fp32 decoder forked into four samples: launches and latency
        {"name": "fork_tiny", "kind": "reorder", "dtype": "fp32", "layers": 2, "heads": 4, "head_dim": 64, "batch": 4,
         "ctx": 60, "slots": 128, "first": 0, "map": "fork"},
        # eight samples of a 1013-token prompt that share it: only its last, partly filled page is copied
        {"name": "fork_tail_7b", "kind": "reorder", "dtype": "bf16", "layers": 8, "heads": 32, "head_dim": 128,
         "batch": 8, "ctx": 1013, "slots": 1280, "first": 1013, "map": "fork"},
        # eight beams after a step, the prompt's 512 slots shared: most follow another beam, one has ended
        {"name": "beams_7b", "kind": "reorder", "dtype": "bf16", "layers": 8, "heads": 32, "head_dim": 128, "batch": 8,
         "ctx": 790, "slots": 1024, "first": 512, "map": "beams"},
        # a serving batch of 16 long sequences: the rows of finished ones are filled from the end of the batch
        {"name": "compact_13b", "kind": "reorder", "dtype": "bf16", "layers": 4, "heads": 40, "head_dim": 128,
         "batch": 16, "ctx": 4000, "slots": 4160, "first": 0, "map": "compact"},
        # four samples of a short prompt, tiny fp32 decoder, k = 5: launches and latency
        {"name": "shared_tiny", "kind": "attention", "dtype": "fp32", "heads": 4, "head_dim": 64, "groups": 1, "n": 4,
         "q": 6, "prefix": 64, "own": 20, "tree": 0},
        # the draft or verify block (k = 5) of eight samples of a 1024-token prompt
        {"name": "shared_7b_n8_q6", "kind": "attention", "dtype": "bf16", "heads": 32, "head_dim": 128, "groups": 1,
         "n": 8, "q": 6, "prefix": 1024, "own": 150, "tree": 0},
        # plain one-token steps of two prompts' samples, ragged, prefixes that end inside a page
        {"name": "shared_7b_2x8_q1", "kind": "attention", "dtype": "bf16", "heads": 32, "head_dim": 128, "groups": 2,
         "n": 8, "q": 1, "prefix": 2011, "own": 300, "tree": 0},
        # four questions of 150 tokens each behind one 2000-token instruction: a prefill block
        {"name": "shared_7b_prefill", "kind": "attention", "dtype": "bf16", "heads": 32, "head_dim": 128, "groups": 1,
         "n": 4, "q": 150, "prefix": 2000, "own": 0, "tree": 0},
        # sixteen samples over a repository-long context, k = 10, 13B heads
        {"name": "shared_13b_16k", "kind": "attention", "dtype": "bf16", "heads": 40, "head_dim": 128, "groups": 1,
         "n": 16, "q": 11, "prefix": 16384, "own": 400, "tree": 0},
        # the log probabilities of a batch-1 loop's tokens with five alternatives (k = 5)
        {"name": "logprobs_b1", "kind": "logprobs", "batch": 1, "q": 6, "vocab": 32016, "n_top": 5, "T": 1.0,
         "ban": 0},
        # a batch of samples at temperature 0.8 over a large vocabulary, twenty alternatives, banned ids
        {"name": "logprobs_128k", "kind": "logprobs", "batch": 16, "q": 6, "vocab": 128256, "n_top": 20, "T": 0.8,
         "ban": 300},
        # a 2047-token prompt scored token by token
        {"name": "logprobs_prompt", "kind": "logprobs", "batch": 1, "q": 2047, "vocab": 32016, "n_top": 1, "T": 1.0,
         "ban": 0},
    ]


HEADS = [(32, 128, "bf16"), (32, 128, "bf16"), (40, 128, "bf16"), (8, 64, "bf16"), (4, 64, "fp32"), (2, 128, "fp32")]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["reorder", "attention", "attention", "attention", "logprobs", "logprobs"])
    if kind == "logprobs":
        vocab = rng.choice([1000, 1024, 32000, 32016, 32016, 32017, 50257, 128256])
        rows = _log_int(rng, 1, min(2000, 60_000_000 // vocab))
        batch = rng.choice([b for b in (1, 1, 2, 3, 4, 8, 16, 24) if b <= rows])
        return {"kind": "logprobs", "batch": batch, "q": rows // batch, "vocab": vocab,
                "n_top": rng.choice([0, 1, 2, 5, 8, 20, 32]), "T": rng.choice([0.2, 0.8, 1.0, 1.0, 1.3]),
                "ban": rng.choice([0, 0, 1, vocab // 2])}
    heads, dh, dtype = rng.choice(HEADS)
    if kind == "reorder":
        batch = _log_int(rng, 2, 24)
        layers = rng.randint(1, 8)
        most = 650_000_000 // (layers * batch * heads * dh)
        ctx = _log_int(rng, 20, min(4000, most))
        return {"kind": "reorder", "dtype": dtype, "layers": layers, "heads": heads, "head_dim": dh, "batch": batch,
                "ctx": ctx, "slots": ctx + rng.randint(1, 200), "first": rng.choice([0, 0, ctx // 3, ctx - 5, ctx]),
                "map": rng.choice(["fork", "beams", "compact"])}
    groups = rng.choice([1, 1, 1, 2, 3])
    if rng.random() < 0.2:   # a prefill block behind the prefix
        n, q, tree = rng.randint(2, 6), _log_int(rng, 65, 300), 0
        prefix, mine = _log_int(rng, 20, min(4000, 2_500_000 // (groups * n * q))), rng.choice([0, 0, 100])
    else:
        n = _log_int(rng, 2, 32 // groups)
        q = rng.randint(1, 16)
        tree = 2 if q >= 3 and q % 2 == 1 and rng.random() < 0.4 else 0
        prefix, mine = _log_int(rng, 10, 16000 // groups), _log_int(rng, 1, 1000)
        q = q if n * groups * q <= 170 else 1
        tree = tree if q > 1 else 0
    return {"kind": "attention", "dtype": dtype, "heads": heads, "head_dim": dh, "groups": groups, "n": n, "q": q,
            "prefix": prefix, "own": mine, "tree": tree}


# ------------------------------------------------------------------ inputs (from the seed alone)
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _pages(n):
    return -(-n // PAGE)


def _slots(n):
    return PAGE * _pages(n)


def _map(case):
    """Where each sequence continues from (-1: its slots are freed).  Sources stay in place, so that a repeated pass
    moves the same pages."""
    n = case["batch"]
    if case["map"] == "fork":
        return [0] * n
    if case["map"] == "compact":   # every third sequence has finished; the last ones take the lowest free rows
        src, last = list(range(n)), n - 1
        for b in range(n):
            if b % 3 == 1:
                while last % 3 == 1:
                    last -= 1
                if b >= last:
                    break
                src[b] = last
                last -= 1
        return src
    src = [0 if b % 2 else b - b % 4 for b in range(n)]   # beams
    if n > 3:
        src[3] = -1
    return src


def _lens(case):
    return [max(1, case["ctx"] - 19 * b) for b in range(case["batch"])]


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


def _cache(case, g):
    """K and V of every layer, sequence and head, [layers, batch, heads, slots, head_dim]: committed slots random, the
    rest zero."""
    shape = (case["layers"], case["batch"], case["heads"], _slots(case["slots"]), case["head_dim"])
    free = torch.arange(shape[3], device="cuda") >= torch.tensor(_lens(case), device="cuda")[:, None]
    kv = []
    for _ in range(2):
        t = _randn(shape, _dtype(case), g)
        for layer in t:
            layer.masked_fill_(free[:, None, :, None], 0)
        kv.append(t)
    return kv


def _prefixes(case):
    return [max(1, case["prefix"] - 45 * i) for i in range(case["groups"])]


def _owns(case):
    """Committed slots of each sequence behind its prefix: ragged, the longest first."""
    return [case["own"] - 13 * b % (case["own"] + 1) for b in range(case["groups"] * case["n"])]


def _tree_mask(q, width):
    """Ancestor masks of a draft tree: root, the chain, then the other candidates of each depth as leaves."""
    k = (q - 1) // width
    mask = [1] + [(1 << (j + 1)) - 1 for j in range(1, k + 1)]
    for j in range(1, k + 1):
        for _ in range(width - 1):
            mask.append(((1 << j) - 1) | (1 << len(mask)))
    return mask


def _shared(case, g):
    """Prefix K and V [groups, heads, prefix, head_dim], the sequences' own (the block's q rows among them)
    [sequences, heads, own + q, head_dim], and the queries [sequences * q, heads * head_dim]."""
    heads, dh, dt = case["heads"], case["head_dim"], _dtype(case)
    batch = case["groups"] * case["n"]
    kp, vp = (_randn((case["groups"], heads, max(_prefixes(case)), dh), dt, g) for _ in range(2))
    ko, vo = (_randn((batch, heads, case["own"] + case["q"], dh), dt, g) for _ in range(2))
    return kp, vp, ko, vo, torch.randn((batch * case["q"], heads * dh), generator=g, device="cuda")


def _visible(case):
    """[sequences, q, own + q]: which of a sequence's own slots each row of its block sees."""
    q, width = case["q"], case["own"] + case["q"]
    rows = torch.ones((q, q), dtype=torch.bool).tril()
    if case["tree"]:
        rows = torch.tensor([[m >> j & 1 for j in range(q)] for m in _tree_mask(q, case["tree"])]).bool()
    see = torch.zeros((case["groups"] * case["n"], q, width), dtype=torch.bool)
    for b, n in enumerate(_owns(case)):
        see[b, :, :n] = True
        see[b, :, n:n + q] = rows
    return see.cuda()


def _logits(case, g):
    """Logits rows, and a token for each: the most probable one, a random one, or -1 (no token in this row)."""
    rows, vocab = case["batch"] * case["q"], case["vocab"]
    x = torch.randn((rows, vocab), generator=g, device="cuda").mul_(4.0)
    x[::3] = (x[::3] * 8).round() / 8   # coarse logits: equal values
    if case["ban"]:
        x[:, vocab - case["ban"]:] = -math.inf
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    pick = torch.rand(rows, generator=g, device="cuda")
    tokens = torch.where(pick < 0.5, x.argmax(-1), tokens)
    return x, torch.where(pick > 0.95, -1, tokens).int()


# ------------------------------------------------------------------ what a program holds before the call
def _context(heads, head_dim, dtype, layers, batch, slots, q, vocab=64):
    """A library context of these heads, slots and vocabulary (the calls here read no weights)."""
    from paper_2403_18647_amd import binding as B
    from paper_2403_18647_amd import synth
    sh = synth.small_shape(n_layers=layers, d_model=heads * head_dim, n_heads=heads, head_dim=head_dim, d_ffn=64,
                           vocab=vocab, n_adaptive=0, dtype=dtype)
    w = [torch.zeros(synth.tensor_shape(sh, n), device="cuda",
                     dtype=torch.float32 if synth.is_gain(n) or dtype == "fp32" else torch.bfloat16)
         for n in synth.tensor_names(sh)]
    return B.Context(B.make_config(sh, batch, slots, q), w)


def prepare(case, seed):
    """Inputs, alike for both forms; the library's cases hold their cache in a context."""
    g = _gen(seed)
    s = {"case": case}
    if case["kind"] == "logprobs":
        rows, top = (case["batch"], case["q"]), (case["batch"], case["q"], case["n_top"])
        s["logits"], s["tokens"] = _logits(case, g)
        if own:
            s["ctx"] = _context(4, 64, "fp32", 1, case["batch"], 32, case["q"], case["vocab"])
            s["out"] = [torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"),
                        torch.empty(top, dtype=torch.int32, device="cuda"), torch.empty(top, device="cuda")]
        return s
    if case["kind"] == "reorder":
        k, v = _cache(case, g)
        s["src"] = torch.tensor(_map(case), dtype=torch.int32, device="cuda")
        if own:
            from paper_2403_18647_amd import binding as B
            s["ctx"] = _context(case["heads"], case["head_dim"], case["dtype"], case["layers"], case["batch"],
                                case["slots"], 1)
            s["k"], s["v"], s["lens"] = s["ctx"].cache()
            s["k"].copy_(k)
            s["v"].copy_(v.view(s["v"].shape))
            B.sdsat_set_cache_len(s["ctx"].handle, _lens(case))
        else:
            s["k"], s["v"], s["lens"] = k, v, torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
        return s
    kp, vp, ko, vo, s["q"] = _shared(case, g)
    batch, q, pre, mine = case["groups"] * case["n"], case["q"], _prefixes(case), _owns(case)
    if own:
        from paper_2403_18647_amd import binding as B
        slots = case["prefix"] + case["own"] + q
        s["ctx"] = _context(case["heads"], case["head_dim"], case["dtype"], 1, batch, slots, q)
        k, v, _ = s["ctx"].cache()
        for b in range(batch):
            i, p = b // case["n"], pre[b // case["n"]]
            lo = 0 if b % case["n"] == 0 else p // PAGE * PAGE   # the first of a group holds the prefix
            for t, tp, to in ((k, kp, ko), (v, vp, vo)):
                row = torch.zeros((case["heads"], _slots(slots), case["head_dim"]), dtype=t.dtype, device="cuda")
                row[:, lo:p] = tp[i, :, lo:p]
                row[:, p:p + mine[b] + q] = to[b, :, :mine[b] + q]
                t[0, b].copy_(row.view(t[0, b].shape))
        B.sdsat_set_cache_len(s["ctx"].handle, [pre[b // case["n"]] + mine[b] for b in range(batch)])
        s["prefix"] = pre
        s["mask"] = None
        if case["tree"]:
            s["mask"] = torch.tensor(_tree_mask(q, case["tree"]) * batch, dtype=torch.int64, device="cuda")
        s["out"] = torch.empty((batch * q, case["heads"] * case["head_dim"]), device="cuda")
        return s
    s["kv"] = kp, vp, ko, vo
    s["in_prefix"] = torch.arange(max(pre), device="cuda") < torch.tensor(pre, device="cuda")[:, None]
    s["see"] = _visible(case)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["kind"] == "reorder":
        return _plain_reorder(s, case)
    if case["kind"] == "attention":
        return _plain_attention(s, case)
    return _plain_logprobs(s, case)


def _run_own(s, case):
    from paper_2403_18647_amd import binding as B
    h = s["ctx"].handle
    if case["kind"] == "reorder":
        B.sdsat_kv_reorder(h, case["batch"], s["src"], case["first"])
        return s["k"], s["v"], s["lens"]
    if case["kind"] == "attention":
        B.sdsat_attention_shared(h, 0, case["groups"] * case["n"], case["q"], case["n"], s["prefix"], s["q"],
                                 s["mask"], s["out"])
        return s["out"]
    lp, ent, ids, top = s["out"]
    if case["n_top"]:
        B.sdsat_token_logprobs(h, case["batch"], case["q"], s["logits"], s["tokens"], case["T"], case["n_top"], lp,
                               ent, ids, top)
        return lp, ent, ids, top
    B.sdsat_token_logprobs(h, case["batch"], case["q"], s["logits"], s["tokens"], case["T"], 0, lp, ent, None, None)
    return lp, ent


def _plain_reorder(s, case):
    """Whole pages from the one that holds slot `first`, up to the end of the source's committed slots."""
    lo, hi = case["first"] // PAGE * PAGE, _slots(max(_lens(case)))   # no other page can move
    lens, src = s["lens"], s["src"].long()
    k, v = s["k"][:, :, :, lo:hi], s["v"][:, :, :, lo:hi]
    at = src.clamp(min=0)
    new_len = torch.where(src >= 0, lens[at], 0).int()
    end = (new_len + PAGE - 1) // PAGE * PAGE
    moved = (torch.arange(lo, max(lo, hi), device=k.device) < end[:, None]) & (src >= 0)[:, None]
    moved = moved[None, :, None, :, None]
    k.copy_(torch.where(moved, k[:, at], k))
    v.copy_(torch.where(moved, v[:, at], v))
    lens.copy_(new_len)
    k, v = s["k"], s["v"]
    return k, v.view(k.shape[:3] + (-1, 2, 4, 4, case["head_dim"])), lens


def _plain_attention(s, case):
    """Scores against the prefix once for all sequences of a group and against each one's own slots; one softmax."""
    kp, vp, ko, vo = (t.float() for t in s["kv"])
    groups, n, q, heads, dh = case["groups"], case["n"], case["q"], case["heads"], case["head_dim"]
    x = s["q"].view(groups, n * q, heads, dh).transpose(1, 2) / math.sqrt(dh)
    mine = s["q"].view(groups * n, q, heads, dh).transpose(1, 2) / math.sqrt(dh)
    sp = torch.matmul(x, kp.transpose(2, 3).contiguous())
    sp = sp.masked_fill(~s["in_prefix"][:, None, None, :], -math.inf)
    so = torch.matmul(mine, ko.transpose(2, 3).contiguous()).masked_fill(~s["see"][:, None], -math.inf)

    def per_group(t):   # [groups * n, heads, q, ...] -> [groups, heads, n * q, ...]
        t = t.view((groups, n) + t.shape[1:]).transpose(1, 2)
        return t.reshape((groups, heads, n * q) + t.shape[4:])

    so = per_group(so)
    top = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    ep, eo = torch.exp(sp - top), torch.exp(so - top)
    den = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    eo = eo.view(groups, heads, n, q, -1).transpose(1, 2).reshape(groups * n, heads, q, -1)
    out = (torch.matmul(ep, vp) + per_group(torch.matmul(eo, vo))) / den
    return out.transpose(1, 2).reshape(groups * n * q, heads * dh)


def _plain_logprobs(s, case):
    rows = (case["batch"], case["q"])
    z = s["logits"] / case["T"]
    z = z - z.amax(-1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    logp = z - torch.log(total)
    at = s["tokens"].long()
    lp = torch.where(at < 0, 0.0, logp.gather(1, at.clamp(min=0)[:, None])[:, 0])
    ent = -torch.where(e > 0, e / total * logp, 0.0).sum(-1)
    if not case["n_top"]:
        return lp.view(rows), ent.view(rows)
    ids = torch.sort(s["logits"], dim=-1, descending=True, stable=True)[1][:, :case["n_top"]]
    top = logp.gather(1, ids)
    return lp.view(rows), ent.view(rows), ids.int().view(rows + (-1,)), top.view(rows + (-1,))


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "reorder":
        # each source's moved pages read once, each destination's written once
        e = 2 if case["dtype"] == "bf16" else 4
        page = 2 * case["layers"] * case["heads"] * case["head_dim"] * PAGE * e
        src, lens, first = _map(case), _lens(case), case["first"] // PAGE
        pages = [max(0, _pages(n) - first) for n in lens]
        moved = {b: a for b, a in enumerate(src) if a >= 0 and a != b}
        n = sum(pages[a] for a in set(moved.values())) + sum(pages[a] for a in moved.values())
        return {"bytes": n * page + 12 * case["batch"], "flops": 0}
    if case["kind"] == "attention":
        e = 2 if case["dtype"] == "bf16" else 4
        d, q, batch = case["heads"] * case["head_dim"], case["q"], case["groups"] * case["n"]
        pre, mine = _prefixes(case), _owns(case)
        by = 2 * d * e * (sum(pre) + sum(n + q for n in mine)) + 2 * batch * q * d * 4
        fl = sum(4.0 * d * (q * (pre[b // case["n"]] + mine[b]) + q * (q + 1) / 2) for b in range(batch))
        return {"bytes": by, "flops": fl}
    rows = case["batch"] * case["q"]
    # an exponential, its sum and its weighted sum for each logit
    return {"bytes": rows * (case["vocab"] * 4 + 12 + 8 * case["n_top"]), "flops": 5.0 * rows * case["vocab"]}


# ------------------------------------------------------------------ the same from the definitions in 64 bits
def exact(case, seed):
    g = _gen(seed)
    if case["kind"] == "reorder":   # copies: the values themselves
        k, v = _cache(case, g)
        src, lens = _map(case), _lens(case)
        out_k, out_v = k.clone(), v.clone()
        for b, a in enumerate(src):
            if a >= 0 and a != b:
                lo, hi = case["first"] // PAGE * PAGE, _slots(lens[a])
                if lo < hi:
                    out_k[:, b, :, lo:hi] = k[:, a, :, lo:hi]
                    out_v[:, b, :, lo:hi] = v[:, a, :, lo:hi]
        new = torch.tensor([lens[a] if a >= 0 else 0 for a in src], dtype=torch.int32)
        return out_k, out_v.view(out_v.shape[:3] + (-1, 2, 4, 4, case["head_dim"])), new
    if case["kind"] == "attention":
        kp, vp, ko, vo, x = _shared(case, g)
        heads, dh, n, q = case["heads"], case["head_dim"], case["n"], case["q"]
        pre, mine, see = _prefixes(case), _owns(case), _visible(case)
        x = x.double().view(-1, q, heads, dh)
        out = torch.empty_like(x)
        for b in range(x.shape[0]):   # one sequence at a time over its whole key list
            p, m = pre[b // n], mine[b] + q
            allowed = torch.cat([torch.ones((q, p), dtype=torch.bool, device="cuda"), see[b, :, :m]], 1)
            for h in range(0, heads, 8):
                hs = slice(h, h + 8)
                kk = torch.cat([kp[b // n, hs, :p], ko[b, hs, :m]], 1).double()
                vv = torch.cat([vp[b // n, hs, :p], vo[b, hs, :m]], 1).double()
                sc = torch.matmul(x[b, :, hs].transpose(0, 1).contiguous(), kk.transpose(1, 2).contiguous())
                w = (sc / math.sqrt(dh)).masked_fill(~allowed, -math.inf).softmax(-1)
                out[b, :, hs] = torch.matmul(w, vv).transpose(0, 1)
        return out.view(-1, heads * dh)
    x, tokens = _logits(case, g)
    rows, n_top = (case["batch"], case["q"]), case["n_top"]
    lp, ent, ids, top = [], [], [], []
    for lo in range(0, x.shape[0], 256):
        logp = (x[lo:lo + 256].double() / case["T"]).log_softmax(-1)
        t = tokens[lo:lo + 256].long()
        lp.append(torch.where(t < 0, torch.zeros_like(logp[:, 0]), logp.gather(1, t.clamp(min=0)[:, None])[:, 0]))
        ent.append(torch.special.entr(logp.exp()).sum(-1))
        i = torch.sort(-x[lo:lo + 256], dim=-1, stable=True)[1][:, :n_top]
        ids.append(i.int())
        top.append(logp.gather(1, i))
    lp, ent = torch.cat(lp).view(rows), torch.cat(ent).view(rows)
    if not n_top:
        return lp, ent
    return lp, ent, torch.cat(ids).view(rows + (n_top,)), torch.cat(top).view(rows + (n_top,))
