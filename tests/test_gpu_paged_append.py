"""Appending to a paged cache against its definition in 64 bits."""
import math

import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paged_helpers import TYPES, Call, assert_within, half_step   # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def frequencies(rot, base=1e6, scaling="none", factor=8.0, ctx=16384.0, low=1.0, high=4.0):
    f = []
    for j in range(rot // 2):
        x = base ** (-2 * j / rot)
        if scaling == "linear":
            x /= factor
        elif scaling == "ntk":
            x = (base * factor ** (rot / (rot - 2))) ** (-2 * j / rot)
        elif scaling == "parts":
            turns = ctx * x / (2 * math.pi)
            share = min(1.0, max(0.0, (turns - low) / (high - low)))
            x = x * share + x / factor * (1 - share)
        f.append(x)
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def turned(x, pos, layout, rot, freq, mscale):
    """x [rows, heads, dh] in 64 bits, rotated; and the size of what was added."""
    x = x.clone()
    size = x.abs()
    if rot:
        a, c = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        w = pos.double()[:, None] * freq
        cos, sin = (torch.cos(w) * mscale)[:, None], (torch.sin(w) * mscale)[:, None]
        p, r = x[..., a].clone(), x[..., c].clone()
        x[..., a], x[..., c] = p * cos - r * sin, r * cos + p * sin
        size[..., a] = size[..., c] = (p.abs() + r.abs()) * abs(mscale)
    return x, size


def append(c, xtype, layout="half", rot=None, scaling="none", base=1e6, mscale=1.0, gains=(None, None), eps=1e-5, pos=None,
           scale=1.0, rope=True):
    """A call with its results against the definition: q, the new slots, and everything else as it was.

    Half a step of the type; in float: dh / 2 + 4 roundings of the norm, 6 of the products, and the sines' error, 2.3e-8 of the
    angle's reduction, a rounding of 16 roundings of 2^-24 for the functions."""
    rot = c.dh if rot is None else rot
    x = c.randn((c.rows, (c.heads + 2 * c.kv) * c.dh), TYPES[xtype], scale)
    q = torch.full((c.rows, c.heads * c.dh), 5.0, dtype=c.dtype, device="cuda")
    k0, v0 = c.k.clone(), c.v.clone()
    r = B.sdsat_rope_init(layout, rot, base, scaling, 8.0, 16384.0, 1.0, 4.0, mscale) if rope else None
    B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, r, pos, gains[0], gains[1], eps, q)
    B.sdsat_paged_status(c.handle)
    at = torch.cat([torch.arange(cached, cached + n) for n, cached in c.seqs]).cuda() if pos is None else pos[:c.start[-1]]
    xd = x.double().view(c.rows, -1, c.dh)[:c.start[-1]]
    parts = []
    for lo, hi, gain in ((0, c.heads, gains[0]), (c.heads, c.heads + c.kv, gains[1])):
        t = xd[:, lo:hi]
        if gain is not None:
            t = t / (t.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
        t, size = turned(t, at, layout, rot if rope else 0, frequencies(rot, base, scaling), mscale)
        parts.append((t, half_step(c.dtype) * t.abs() + size * ((c.dh / 2 + 26) * 2.0 ** -24 + 2.3e-8) * 1.01 + 1e-30))
    (wq, tq), (wk, tk) = parts
    n = c.start[-1]
    assert_within(q[:n].view(n, c.heads, c.dh), wq, tq, "q")
    assert (q[n:] == 5).all()
    wv = xd[:, c.heads + c.kv:]
    k1, v1 = c.k.clone(), c.v.clone()
    for b, (new, cached) in enumerate(c.seqs):
        if not new:
            continue
        k, v = c.get(b, cached, cached + new)
        rows = slice(c.start[b], c.start[b + 1])
        assert_within(k, wk[rows], tk[rows], "k")
        assert torch.equal(v.double(), wv[rows].to(c.dtype).double()), "v"
        page, place = c.slots(b, cached, cached + new)
        old_k = k0[page, :, place]
        k1[page, :, place] = old_k
        from paged_helpers import place as in_page
        v1[page, :, :, in_page(place)] = v0[page, :, :, in_page(place)]
    assert torch.equal(k1.view(torch.uint8), k0.view(torch.uint8)), "other slots of K"
    assert torch.equal(v1.view(torch.uint8), v0.view(torch.uint8)), "other slots of V"
    return q


RAGGED = [[(1, 0)], [(1, 31), (1, 32), (0, 7), (1, 95)], [(6, 90), (6, 30)], [(8, 24), (9, 31), (33, 0), (64, 32)],
          [(130, 17), (1, 64), (0, 0), (200, 1), (3, 62)]]


@pytest.mark.parametrize("dtype,xtype,heads,kv,dh", [("bf16", "bf16", 8, 2, 128), ("bf16", "fp32", 3, 3, 128),
                                                     ("bf16", "bf16", 7, 1, 64), ("fp32", "fp32", 4, 4, 64),
                                                     ("fp32", "bf16", 6, 2, 128)])
@pytest.mark.parametrize("seqs", RAGGED, ids=lambda s: "_".join(f"{n}at{c}" for n, c in s))
def test_against_definition(dtype, xtype, heads, kv, dh, seqs):
    print(f"case {dtype} {xtype} {heads}/{kv}x{dh} {seqs}", flush=True)
    c = Call(seqs, heads, kv, dh, dtype, spare=3)
    gains = tuple(1 + 0.1 * c.randn((dh,), torch.float32) for _ in range(2))
    append(c, xtype)
    append(c, xtype, gains=gains, layout="interleaved")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [0, 8, 24, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "parts"])
def test_layouts_and_scalings(layout, rot, scaling):
    """Parts of the head, far and negative positions (given ones), cosines and sines with a factor."""
    print(f"case {layout} {rot} {scaling}", flush=True)
    c = Call([(40, 3), (1, 700)], 4, 2, 128, "fp32", spare=2)
    append(c, "fp32", layout, rot, scaling)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (c.rows,), generator=c.g, device="cuda", dtype=torch.int64).int()
    pos[:8] = torch.tensor([0, 1, -1, 10 ** 6, 2 ** 24 + 1, 2 ** 30, 2 ** 31 - 1, -2 ** 31])
    # at 2^31 turns a double's half step is 2^-22 of a radian for the fastest pair: the test's own angle is that far off
    far = append_far(c, layout, rot, scaling, pos)
    assert far


def append_far(c, layout, rot, scaling, pos):
    """Positions of any size: rotations keep lengths, and agree with 64 bits to the angle's error there."""
    x = c.randn((c.rows, (c.heads + 2 * c.kv) * c.dh), torch.float32)
    q = torch.zeros((c.rows, c.heads * c.dh), device="cuda")
    r = B.sdsat_rope_init(layout, rot, 1e6, scaling, 8.0, 16384.0, 1.0, 4.0, 1.25)
    B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, r, pos, None, None, 0.0, q)
    n = c.start[-1]
    xd = x.double().view(c.rows, -1, c.dh)[:n, :c.heads]
    want, size = turned(xd, pos[:n], layout, rot, frequencies(rot, 1e6, scaling), 1.25)
    angle = 4 * 2.0 ** -53 * pos[:n].double().abs()[:, None, None]   # of the products with a frequency (<= 1) on both sides
    assert_within(q[:n].view(n, c.heads, c.dh), want, size * (32 * 2.0 ** -24 + 2.3e-8 + angle) + 1e-30, "far")
    return True


def test_one_gain_alone_eps_and_no_rotation():
    c = Call([(20, 5)], 4, 2, 64, "bf16")
    g = 1 + 0.1 * c.randn((64,), torch.float32)
    append(c, "fp32", gains=(g, None), eps=0.5, scale=0.01)
    append(c, "bf16", gains=(None, g), rope=False)


def test_zero_rows_and_zero_columns():
    """A head of zeros is normalised with eps; infinities stay what they are elsewhere."""
    c = Call([(2, 5)], 2, 1, 64, "fp32")
    x = torch.zeros((2, 256), device="cuda")
    x[1, 64:128] = 1e30   # mean of squares past float's range: 1 / inf
    q = torch.full((2, 128), 3.0, device="cuda")
    g = torch.ones(64, device="cuda")
    B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, None, None, g, g, 1e-6, q)
    assert (q == 0).all()


def test_strided_rows():
    c = Call([(9, 30), (1, 5)], 4, 2, 64, "bf16", spare=1)
    wide = c.randn((c.rows, 8 + 512 + 24))
    x = wide[:, 8:520]
    q = torch.full((c.rows, 288), 5.0, dtype=c.dtype, device="cuda")
    B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, None, None, None, None, 0.0, q[:, 16:272])
    assert torch.equal(q[:10, 16:272], x[:10, :256])
    assert (q[10] == 5).all() and (q[:, :16] == 5).all() and (q[:, 272:] == 5).all()
    k, v = c.get(0, 30, 39)
    assert torch.equal(k.reshape(9, 128), x[:9, 256:384]) and torch.equal(v.reshape(9, 128), x[:9, 384:])


def test_numbers_that_do_not_fit_are_reported():
    c = Call([(2, 40), (3, 50), (1, 7)], 4, 2, 64)
    x = c.randn((c.rows, 512))
    q = torch.zeros((c.rows, 256), dtype=c.dtype, device="cuda")
    good = c.d_len.clone(), c.d_start.clone(), c.pages.clone()
    for what, t, at, value in [("len", c.d_len, 1, -1), ("len", c.d_len, 1, 2 ** 31 - 1), ("len", c.d_len, 1, 51),
                               ("start", c.d_start, 1, 4), ("start", c.d_start, 2, 1), ("start", c.d_start, 3, 99),
                               ("start", c.d_start, 0, -2), ("page", c.pages, (1, 1), c.n_pages),
                               ("page", c.pages, (1, 1), -1)]:
        print(what, at, value, flush=True)
        t[at] = value
        k0, v0 = c.k.clone(), c.v.clone()
        B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, None, None, None, None, 0.0, q)
        with pytest.raises(B.SdsatError) as e:
            B.sdsat_paged_status(c.handle)
        assert e.value.code == -6 and ("page" in str(e.value)) == (what == "page")
        if what != "start":   # of the pool only what the others append has changed
            for b, first, n in ((0, 40, 2), (2, 7, 1)):
                page, place = c.slots(b, first, first + n)
                from paged_helpers import place as in_page
                c.k[page, :, place] = k0[page, :, place]
                c.v[page, :, :, in_page(place)] = v0[page, :, :, in_page(place)]
            assert torch.equal(c.k, k0) and torch.equal(c.v, v0)
        for t, g in zip((c.d_len, c.d_start, c.pages), good):
            t.copy_(g)
    # entries that no new slot needs are not looked at
    c.pages[1, 0] = -1
    B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, None, None, None, None, 0.0, q)
    B.sdsat_paged_status(c.handle)


def test_more_than_64_sequences():
    append(Call([(1 + 3 * (b % 5 == 2), 37 * b % 500) for b in range(200)] + [(40, 3)], 4, 2, 64), "bf16")


def test_pools_past_4_gib():
    c = Call([(1, 70), (100, 10)], 16, 8, 128, n_pages=70000, extra_pages=0, fill=0.0)
    c.pages.copy_(torch.arange(69999, 69999 - c.pages.numel(), -1).view(c.pages.shape))
    x = c.randn((c.rows, 32 * 128))
    q = torch.zeros((c.rows, 2048), dtype=c.dtype, device="cuda")
    B.sdsat_paged_append(c.handle, c.batch, c.k, c.v, x, None, None, None, None, 0.0, q)
    for b, (n, cached) in enumerate(c.seqs):
        k, v = c.get(b, cached, cached + n)
        rows = slice(c.start[b], c.start[b + 1])
        assert torch.equal(k.reshape(n, -1), x[rows, 2048:2048 + 1024]) and torch.equal(v.reshape(n, -1), x[rows, 2048 + 1024:])
    assert not c.k[:60000].any() and not c.v[:60000].any()
