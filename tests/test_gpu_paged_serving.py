"""The paged cache's calls together, as a server makes them: linear layers, appending, attention, logit rules and
verification in turn, captured and replayed, on several streams, beside the contiguous cache; and what handles refuse."""
import numpy as np
import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from operator_helpers import context, device_error   # noqa: E402
from paged_helpers import Call, assert_within, half_step, place   # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def ints(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class Layer:
    """One attention layer with 4 query heads over 2 key heads of 64, norms by head, and an output layer, behind the
    library's linear layers."""
    H, KV, DH, D, VOCAB = 4, 2, 64, 192, 500

    def __init__(self, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(5)
        self.code = B.DTYPE_BF16 if dtype == torch.bfloat16 else B.DTYPE_FP32
        self.dtype = dtype
        self.w = {}
        for name, n, k in (("qkv", (self.H + 2 * self.KV) * self.DH, self.D), ("o", self.VOCAB, self.H * self.DH)):
            w = (torch.randn((n, k), generator=self.g, device="cuda") / k ** 0.5).to(dtype)
            packed = torch.empty(B.sdsat_linear_packed_bytes(self.code, n, k), dtype=torch.uint8, device="cuda")
            B.sdsat_linear_pack(self.code, n, k, w, packed)
            self.w[name] = (n, k, packed)
        self.gain = 1 + 0.1 * torch.randn((2, self.DH), generator=self.g, device="cuda")
        self.rope = B.sdsat_rope_init("half", 32, 1e4, "linear", 4.0)

    def linear(self, name, x, y):
        n, k, packed = self.w[name]
        scratch = torch.empty(B.sdsat_linear_scratch_bytes(x.shape[0], n, k), dtype=torch.uint8, device="cuda")
        B.sdsat_linear(self.code, x.shape[0], n, k, x, packed, y, scratch)

    def step(self, c, x, bufs, ctx, batch, q, rules, seed):
        """x [rows, D] -> logits of the rows, the adjusted ones, their tokens."""
        qkv, qr, att, logits, adjusted, tokens, accepted, pos0 = bufs
        self.linear("qkv", x, qkv)
        B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, qkv, self.rope, None, self.gain[0], self.gain[1], 1e-6, qr)
        B.sdsat_paged_attention(c.handle, c.batch, c.k, c.v, qr, None, 0, 0.0, att)
        self.linear("o", att, logits)
        B.sdsat_adjust_logits(ctx.handle, batch, q, logits, rules, adjusted)
        B.sdsat_verify_nucleus(ctx.handle, batch, q, adjusted, None, 0.9, 0.95, 40, seed, pos0, tokens, accepted)

    def buffers(self, rows, batch):
        f = lambda n: torch.zeros((rows, n), device="cuda")
        return (f((self.H + 2 * self.KV) * self.DH), torch.zeros((rows, self.H * self.DH), dtype=self.dtype, device="cuda"),
                f(self.H * self.DH), f(self.VOCAB), f(self.VOCAB), ints([0] * rows), ints([0] * batch), ints([7] * batch))


def rule_set(batch, q, vocab, g):
    return dict(history=torch.randint(0, vocab, (batch, 30), generator=g, device="cuda").int(), history_len=ints([30] * batch),
                prompt_len=ints([10] * batch), tokens=torch.randint(0, vocab, (batch, q), generator=g, device="cuda").int(),
                penalties=torch.tensor([[1.2], [0.3], [0.1]], device="cuda").repeat(1, batch),
                allowed=torch.randint(-2 ** 31, 2 ** 31, (batch * q, (vocab + 31) // 32), generator=g, device="cuda").int())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_steps_of_a_server(dtype):
    """Prompts in pieces, then blocks, then single tokens, of three sequences that start at different times; each call's
    output against its definition on what the call before left."""
    q = {"bf16": 4, "fp32": 4}[dtype]
    lengths = [0, 0, 0]
    layer = None
    keep = None
    for step, news in enumerate([[20, 0, 0], [30, 12, 0], [q, q, q], [1, 1, 1], [q, q, q]]):
        c = Call([(n, l) for n, l in zip(news, lengths)], Layer.H, Layer.KV, Layer.DH, dtype, pages_width=4, n_pages=12,
                 max_batch=3, max_ctx=128, max_rows=64)
        layer = layer or Layer(c.dtype)
        if keep is None:
            keep = (c.k, c.v, torch.randperm(12, generator=layer.g, device="cuda").int().view(3, 4))
        c.k, c.v, c.pages = keep
        c.describe()
        x = torch.randn((c.rows, Layer.D), generator=layer.g, device="cuda")
        uniform = news[0] == news[2]
        batch, rows = (3, news[0]) if uniform else (1, c.rows)
        ctx = context(batch=batch, q=max(rows, 1), vocab=Layer.VOCAB)
        rs = rule_set(batch, rows, Layer.VOCAB, layer.g)
        bufs = layer.buffers(c.rows, batch)
        layer.step(c, x, bufs, ctx, batch, rows, B.logit_rules(**rs), step)
        B.sdsat_paged_status(c.handle)
        assert device_error(ctx) == 0
        qkv, qr, att, logits, adjusted, tokens = bufs[:6]
        # appended: what the call's rows say
        new = qkv.double().view(c.rows, -1, Layer.DH)
        at = 0
        for b, (n, l) in enumerate(c.seqs):
            k, v = c.get(b, l, l + n)
            kk = new[at:at + n, Layer.H:Layer.H + Layer.KV]
            kk = kk / (kk.square().mean(-1, keepdim=True) + 1e-6).sqrt() * layer.gain[1].double()
            w = (torch.arange(l, l + n, device="cuda").double()[:, None] * 1e4 ** (-torch.arange(16, device="cuda").double() / 16) / 4)[:, None]
            a, s = kk[..., :16].clone(), kk[..., 16:32].clone()
            kk[..., :16], kk[..., 16:32] = a * w.cos() - s * w.sin(), s * w.cos() + a * w.sin()
            size = kk.abs()
            size[..., :16] = size[..., 16:32] = a.abs() + s.abs()
            assert_within(k, kk, half_step(c.dtype) * kk.abs() + size * (58 * 2.0 ** -24 + 2.3e-8) * 1.01 + 1e-30, "k")
            assert torch.equal(v.double(), new[at:at + n, Layer.H + Layer.KV:].to(c.dtype).double())
            at += n
        assert_within(att, *c.expected(qr, u_out=2.0 ** -24), what="attention")
        # a token of each row is one that the grammar allows
        bits = rs["allowed"][torch.arange(c.rows), tokens.long() // 32] >> (tokens % 32) & 1
        assert (bits == 1).all() and (adjusted[torch.arange(c.rows), tokens.long()] > -float("inf")).all()
        lengths = [l + n for l, n in zip(lengths, news)]
        ctx.close()


def test_a_captured_step():
    """The whole step in one graph: replayed with other inputs and lengths, with eager steps on the same buffers between;
    every replay gives the eager step's bits."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        batch, q = 3, 4
        c = Call([(q, 40), (q, 10), (q, 90)], Layer.H, Layer.KV, Layer.DH, n_pages=14, max_ctx=128)
        c.max_len = 128
        c.pages = torch.randperm(14, generator=c.g, device="cuda").int()[:12].view(3, 4).contiguous()
        c.describe()
        layer = Layer(c.dtype)
        ctx = context(batch=batch, q=q, vocab=Layer.VOCAB)
        rs = rule_set(batch, q, Layer.VOCAB, layer.g)
        rules = B.logit_rules(**rs)
        x = torch.randn((c.rows, Layer.D), generator=layer.g, device="cuda")
        bufs = layer.buffers(c.rows, batch)
        layer.step(c, x, bufs, ctx, batch, q, rules, 1)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            layer.step(c, x, bufs, ctx, batch, q, rules, 1)
        for i in range(4):
            x.copy_(torch.randn(x.shape, generator=layer.g, device="cuda"))
            c.d_len.copy_(ints([40 + 5 * i, 3 * i, 124 - i]))
            rs["history_len"].copy_(ints([30 - i, i, 0]))
            layer.step(c, x, bufs, ctx, batch, q, rules, 1)
            eager = [t.clone() for t in bufs] + [c.k.clone(), c.v.clone()]
            for t in bufs[:6]:
                t.zero_()
            graph.replay()
            stream.synchronize()
            for a, b in zip(list(bufs) + [c.k, c.v], eager):
                assert torch.equal(a, b)
        B.sdsat_paged_status(c.handle)
        assert device_error(ctx) == 0
        ctx.close()


def test_handles_on_two_streams_at_once():
    calls, want = [], []
    for i, seqs in enumerate([[(1, 1800), (1, 900)], [(70, 500), (3, 20)]]):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            c = Call(seqs, 8, 2, 64, seed=i)
            q = c.randn((c.rows, 512))
            out = torch.zeros_like(q)
            want.append(c.attend(q))
            calls.append((s, c, q, out))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, c, q, out in calls:
            c.attend(q, out=out)   # each on its handle's stream, whichever is the current one
    torch.cuda.synchronize()
    for (s, c, q, out), w in zip(calls, want):
        assert torch.equal(out, w)


def test_pages_of_the_contiguous_cache():
    """Whole pages taken from a context's cache as they are: the same attention from both, and from pages shared by two."""
    lens, q = [70, 33], 3
    ctx = context(heads=4, head_dim=64, batch=2, slots=128, q=q, vocab=64)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = max(lens) + q
    k, v = (torch.randn((2, n, 4, 64), generator=g, device="cuda") for _ in range(2))
    pos = torch.arange(n, device="cuda").int().repeat(2, 1).contiguous()
    B.sdsat_kv_write(ctx.handle, 0, 2, n, k, v, pos)
    B.sdsat_set_cache_len(ctx.handle, lens)
    qin = torch.randn((2 * q, 256), generator=g, device="cuda")
    there = torch.empty_like(qin)
    B.sdsat_attention(ctx.handle, 0, 2, q, qin, None, there)
    c = Call([(q, l) for l in lens], 4, 4, 64, "fp32", n_pages=9)
    ck, cv, _ = ctx.cache()
    for b in range(2):
        for i in range(-(-(lens[b] + q) // 32)):
            page = int(c.pages[b, i])
            c.k[page] = ck[0, b, :, 32 * i:32 * i + 32]
            # [heads, a, g, r, dh] to [heads, dh, 8g + 4a + r]
            c.v[page] = cv[0, b, :, i].permute(0, 4, 2, 1, 3).reshape(4, 64, 32)
    here = c.attend(qin)
    want, tol = c.expected(qin)
    assert_within(here, want, tol)
    assert_within(there, want, tol)
    for b in range(2):
        kk, vv = c.get(b, 0, lens[b] + q)
        assert torch.equal(kk, k[b, :lens[b] + q]) and torch.equal(vv, v[b, :lens[b] + q])
    ctx.close()


def test_calls_that_are_refused():
    c = Call([(3, 40), (70, 5)], 4, 2, 64, spare=1)
    x, qo = c.randn((c.rows, 512)), c.randn((c.rows, 256))
    m = torch.zeros(c.rows, dtype=torch.int64, device="cuda")

    def desc(**kw):
        a = dict(start=c.d_start, length=c.d_len, pages=c.pages, rows=c.rows, max_q=70, max_len=75)
        a.update(kw)
        return B.paged_batch(**a)

    many = dict(start=ints([0] * 4), length=ints([0] * 3), pages=torch.zeros((3, c.width), dtype=torch.int32, device="cuda"))
    for kw, code in [(dict(rows=-1), -1), (dict(rows=c.rows + 1), -4), (dict(max_q=-1), -1), (dict(max_q=c.rows + 1), -1),
                     (dict(max_len=69), -1), (dict(max_len=-5), -1), (dict(max_len=10 ** 6), -4), (many, -4),
                     (dict(pages=c.pages[:, :2]), -4 if c.pages.stride(0) == 2 else None)]:
        if code is None:   # a narrower view of the same table keeps its stride
            continue
        for call in (lambda d: B.sdsat_paged_append(c.handle, d, c.k, c.v, x, q_out=qo),
                     lambda d: B.sdsat_paged_attention(c.handle, d, c.k, c.v, qo, out=qo)):
            with pytest.raises(B.SdsatError) as e:
                call(desc(**kw))
            assert e.value.code == code, (kw, e.value)
    narrow = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_paged_append(c.handle, desc(pages=narrow), c.k, c.v, x, q_out=qo)
    assert e.value.code == -4

    lib = B.lib()
    d = desc()
    import ctypes
    ref = ctypes.byref(d)
    p = lambda t: t.data_ptr()

    def append(k=p(c.k), v=p(c.v), xx=p(x), code=1, ldx=512, rope=None, eps=0.0, q=p(qo), ldq=256):
        return lib.sdsat_paged_append(c.handle, ref, k, v, xx, code, ldx, rope, None, None, None, eps, q, ldq)

    def attend(k=p(c.k), v=p(c.v), q=p(qo), ldq=256, mask=None, window=0, scale=0.0, out=p(qo), code=1, ldo=256):
        return lib.sdsat_paged_attention(c.handle, ref, k, v, q, ldq, mask, window, scale, out, code, ldo)

    far = B.sdsat_rope_init("half", 128)
    odd = B.sdsat_rope()
    odd.layout = 5
    for kw in (dict(k=None), dict(v=None), dict(xx=None), dict(q=None), dict(code=2), dict(ldx=504), dict(ldx=516), dict(ldq=248),
               dict(ldq=260), dict(eps=-1.0), dict(eps=float("nan")), dict(xx=p(x) + 8), dict(k=p(c.k) + 4),
               dict(rope=ctypes.byref(far)), dict(rope=ctypes.byref(odd))):
        assert append(**kw) == -1, kw
    for kw, code in [(dict(k=None), -1), (dict(v=None), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(code=3), -1),
                     (dict(ldq=248), -1), (dict(ldo=252), -1), (dict(window=-1), -1), (dict(scale=-1.0), -1),
                     (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(q=p(qo) + 2), -1),
                     (dict(mask=p(m)), -5)]:
        assert attend(**kw) == code, kw
    small = Call([(3, 40)], 4, 2, 64)
    with pytest.raises(B.SdsatError) as e:
        small.attend(small.randn((3, 256)), mask=m[:3], window=4)
    assert e.value.code == -5
    single = Call([(3, 40)], 4, 2, 64, "fp32")
    assert lib.sdsat_paged_attention(single.handle, ctypes.byref(single.batch), p(single.k), p(single.v), p(x), 256, None, 0, 0.0,
                                     p(x), 1, 256) == -1   # bf16 outputs of an fp32 cache
    # nothing to do is no error
    none = Call([(0, 40), (0, 0)], 4, 2, 64, spare=4)
    qn = torch.full((4, 256), 3.0, dtype=none.dtype, device="cuda")
    B.sdsat_paged_append(none.handle, none.batch, none.k, none.v, none.randn((4, 512)), q_out=qn)
    assert (none.attend(qn, out=qn) == 3).all()
    B.sdsat_paged_status(none.handle)

    ctx = context(batch=1, q=70, vocab=64)
    z = torch.zeros((70, 64), device="cuda")
    h = torch.zeros((1, 8), dtype=torch.int32, device="cuda")
    for q, kw, code in [(1, dict(history=h), -1), (1, dict(mask=m[:1]), -1), (70, dict(tokens=torch.zeros((1, 70), dtype=torch.int32, device="cuda")), -5),
                        (1, dict(allowed=torch.zeros((1, 1), dtype=torch.int32, device="cuda")), -1),
                        (1, dict(bias=torch.zeros((2, 63), device="cuda")), -1), (71, {}, -4), (0, {}, -1)]:
        with pytest.raises(B.SdsatError) as e:
            B.sdsat_adjust_logits(ctx.handle, 1, q, z, B.logit_rules(**kw), z)
        assert e.value.code == code, (kw, e.value)
    r = B.logit_rules(history=h, history_len=ints([1]))
    r.history_ld = 1 << 24
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_adjust_logits(ctx.handle, 1, 1, z, r, z)
    assert e.value.code == -5
    ctx.close()
