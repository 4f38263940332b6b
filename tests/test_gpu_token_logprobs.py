"""sdsat_token_logprobs against float64: vocabularies of one id to several chunks, rows at odd offsets, ties, banned ids,
NaN and infinities, peaked rows, padded rows, refusals, streams and captured graphs."""
import math

import pytest
import torch

from operator_helpers import context, device_error
from paper_2403_18647_amd import binding as B

pytestmark = pytest.mark.gpu


def call(ctx, batch, q, x, tokens, T=1.0, n_top=0, lp=True, ent=True):
    a = torch.full((batch, q), 7e7, device="cuda") if lp else None
    b = torch.full((batch, q), 7e7, device="cuda") if ent else None
    ids = torch.full((batch, q, n_top), -9, dtype=torch.int32, device="cuda") if n_top else None
    top = torch.full((batch, q, n_top), 7e7, device="cuda") if n_top else None
    B.sdsat_token_logprobs(ctx.handle, batch, q, x, tokens, T, n_top, a, b, ids, top)
    torch.cuda.synchronize()
    return a, b, ids, top


def check(x, tokens, T, n_top, got):
    """A log probability is t - log1p(S): t = (x - max) / T errs by 3 roundings of |t| (1/T, difference, product); a term
    of S by its t (times log2 e, rounded: 3 |t| 2^-24 more) and exp2 (2^-23), its sums by one rounding per addition
    (32 ids per thread, 6 steps in a wave, 4 waves, the chunks: at most 64): together at most (64 + 6 H') 2^-24 relative,
    H' = sum p |t| <= the entropy; log1p and the difference round once each.  The entropy adds the error of
    sum p |t|: the same relative error of each term, and of t itself."""
    lp, ent, ids, top = got
    rows, V = x.shape
    z = x.double() / T
    logp = z.log_softmax(-1)
    p = logp.exp()
    h = torch.special.entr(p).sum(-1)
    logs = -logp.amax(-1)
    rel = (64 + 6 * h) * 2.0 ** -24
    if lp is not None:
        at = tokens.long()
        want = torch.where(at < 0, torch.zeros_like(h), logp.gather(1, at.clamp(min=0)[:, None])[:, 0])
        tol = rel + (want.abs() + 2 * logs) * 2.0 ** -22
        got_lp = lp.view(-1).double()
        same = got_lp == want   # -inf for banned tokens
        assert bool((same | ((got_lp - want).abs() <= tol)).all()), float((got_lp - want).abs()[~same].max())
    if ent is not None:
        tol = rel * (2 + 2 * h) + (h + logs) * 2.0 ** -22
        off = (ent.view(-1).double() - h).abs()
        assert bool((off <= tol).all()), float((off / tol).max())
    if n_top:
        want_ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :n_top]
        assert torch.equal(ids.view(rows, n_top).long(), want_ids)
        want = logp.gather(1, want_ids)
        tol = rel[:, None] + (want.abs() + 2 * logs[:, None]) * 2.0 ** -22
        got_top = top.view(rows, n_top).double()
        same = got_top == want
        assert bool((same | ((got_top - want).abs() <= tol)).all())


def logits(rows, V, seed, scale=4.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, V), generator=g, device="cuda") * scale
    return x, torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("V", [2, 3, 31, 63, 64, 1000, 1023, 8191, 8192, 8193, 8194, 32016, 50257, 128256])
@pytest.mark.parametrize("batch,q", [(1, 1), (3, 5)])
def test_vocabularies(V, batch, q):
    ctx = context(batch=batch, q=q, vocab=V)
    x, tokens = logits(batch * q, V, V)
    for n_top, T in ((0, 1.0), (1, 0.7), (min(V, 5), 1.0), (min(V, 32), 1.9)):
        check(x, tokens, T, n_top, call(ctx, batch, q, x, tokens, T, n_top))
    assert device_error(ctx) == 0
    ctx.close()


def test_many_rows():
    ctx = context(batch=2, q=600, vocab=9001)
    x, tokens = logits(1200, 9001, 1)
    check(x, tokens, 1.0, 3, call(ctx, 2, 600, x, tokens, 1.0, 3))
    ctx.close()


@pytest.mark.parametrize("V", [1024, 1025, 4095, 4097, 5121, 12289, 20483])
@pytest.mark.parametrize("rows", [1, 1100])
def test_ragged_tiles(V, rows):
    """Rows cut into segments whose last is a few ids, and rows of one segment; the largest at both ends of the row and of
    the last tiles."""
    ctx = context(batch=1, q=rows, vocab=V)
    x, tokens = logits(rows, V, V + rows, scale=1.0)
    for i, at in enumerate((0, 1023, 1024, 4095, 4096, V - 1025, V - 1024, V - 5, V - 4, V - 1)):
        if 0 <= at < V:
            x[:, at] = 8.0 + i % 3
    check(x, tokens, 1.0, 12, call(ctx, 1, rows, x, tokens, 1.0, 12))
    ctx.close()


@pytest.mark.parametrize("V,step", [(1000, 1.0), (9000, 8.0), (32016, 3.0), (32016, 0.0)])
def test_ties_go_to_the_lower_id(V, step):
    ctx = context(batch=1, q=4, vocab=V)
    x, tokens = logits(4, V, 2)
    x = (x / step).round() * step if step else torch.zeros_like(x)   # -0 among the values
    x[3] = -x[3].abs()
    check(x, tokens, 1.0, 32, call(ctx, 1, 4, x, tokens, 1.0, 32))
    ctx.close()


@pytest.mark.parametrize("V", [8192, 20000])
def test_values_in_an_order(V):
    """Rising, falling, and all large values in the ids of one group of threads (the most candidates)."""
    ctx = context(batch=1, q=4, vocab=V)
    x = torch.empty((4, V), device="cuda")
    ramp = torch.arange(V, device="cuda") * 1e-3
    x[0], x[1] = ramp, -ramp
    some = (torch.arange(V, device="cuda") % 1024) < 16
    x[2] = torch.where(some, ramp + 20, ramp * 1e-3)
    most = (torch.arange(V, device="cuda") % 1024) < 16 * 31
    x[3] = torch.where(most, ramp + 20, ramp * 1e-3)
    tokens = torch.tensor([0, V - 1, 5, 16], dtype=torch.int32, device="cuda")
    check(x, tokens, 1.0, 32, call(ctx, 1, 4, x, tokens, 1.0, 32))
    ctx.close()


def test_peaked_rows_keep_small_differences():
    """One id with nearly all mass: its log probability is minus the others' mass, far below a float's step at 1."""
    V = 20000
    ctx = context(batch=1, q=3, vocab=V)
    x = torch.full((3, V), -25.0, device="cuda")
    x[0, 3], x[1, 19999], x[2, 8192] = 5.0, 2.0, 0.0
    tokens = torch.tensor([3, 19999, 8192], dtype=torch.int32, device="cuda")
    lp, ent, _, _ = call(ctx, 1, 3, x, tokens)
    logp = x.double().log_softmax(-1)
    want = logp.gather(1, tokens.long()[:, None])[:, 0]
    h = torch.special.entr(logp.exp()).sum(-1)
    # relative now: sums of V equal terms (errors as in check, without the differences of check's absolute bounds)
    rel = (64 + 6 * 30) * 2.0 ** -24 + 2.0 ** -22
    assert bool(((lp.view(-1).double() - want).abs() <= rel * want.abs()).all())
    assert bool(((ent.view(-1).double() - h).abs() <= 2 * rel * h).all())
    ctx.close()


@pytest.mark.parametrize("V", [500, 8200, 32016])
def test_banned_ids(V):
    ctx = context(batch=1, q=5, vocab=V)
    x, tokens = logits(5, V, 3)
    x[0, V // 2:] = -math.inf
    x[1, : V - 3] = -math.inf          # fewer ids left than alternatives
    x[2, 1:] = -math.inf               # one id left
    x[3, ::2] = -math.inf
    x[4, 5] = -3e38
    tokens[0], tokens[1], tokens[2] = V - 1, V - 2, 0   # banned, allowed, certain
    for T in (1.0, 0.2):
        check(x, tokens, T, 8, call(ctx, 1, 5, x, tokens, T, 8))
    assert device_error(ctx) == 0
    ctx.close()


@pytest.mark.parametrize("V", [100, 8193, 32016])
def test_rows_without_a_distribution(V):
    """NaN, +inf, nothing but -inf: NaN results, and the rows beside them are untouched by it."""
    ctx = context(batch=1, q=7, vocab=V)
    x, tokens = logits(7, V, 4)
    x[1, V - 1] = math.nan
    x[2, V // 3] = math.inf
    x[3] = -math.inf
    x[4] = math.nan
    x[5, V - 2:] = math.inf
    lp, ent, ids, top = call(ctx, 1, 7, x, tokens, 1.0, 4)
    for r in (1, 2, 3, 4, 5):
        assert bool(lp[0, r].isnan()) and bool(ent[0, r].isnan()) and bool(top[0, r].isnan().all()), r
    order = torch.sort(x.nan_to_num(-math.inf, math.inf, -math.inf), dim=-1, descending=True, stable=True)[1]
    for r in (1, 2, 3, 5):
        assert torch.equal(ids[0, r].long(), order[r, :4]), r
    assert ids[0, 4].tolist() == [0, 1, 2, 3]
    keep = torch.tensor([0, 6], device="cuda")
    check(x[keep], tokens[keep], 1.0, 4, (lp[0, keep], ent[0, keep], ids[0, keep], top[0, keep]))
    ctx.close()


def test_rows_without_a_token_and_ids_past_the_vocabulary():
    V = 9000
    ctx = context(batch=2, q=3, vocab=V)
    x, tokens = logits(6, V, 5)
    tokens[1] = -1
    tokens[4] = -2147483648
    check(x, tokens, 1.0, 2, call(ctx, 2, 3, x, tokens, 1.0, 2))
    assert device_error(ctx) == 0
    tokens[2] = V
    lp, ent, _, _ = call(ctx, 2, 3, x, tokens, 1.0, 2)
    assert bool(lp[0, 2].isnan()) and not bool(ent.isnan().any()) and int(lp.isnan().sum()) == 1
    assert device_error(ctx) == -6 and device_error(ctx) == 0
    ctx.close()


def test_only_what_is_asked_for():
    V = 9000
    ctx = context(batch=1, q=3, vocab=V)
    x, tokens = logits(3, V, 6)
    lp, ent, ids, top = call(ctx, 1, 3, x, tokens, 1.0, 3)
    assert torch.equal(call(ctx, 1, 3, x, tokens, ent=False)[0], lp)
    assert torch.equal(call(ctx, 1, 3, x, None, lp=False)[1], ent)
    got = call(ctx, 1, 3, x, None, n_top=3, lp=False, ent=False)
    assert torch.equal(got[2], ids) and torch.equal(got[3], top)
    call(ctx, 1, 3, x, None, lp=False, ent=False)
    # rows do not depend on the rows beside them, and a row's place in memory (odd offsets) does not matter
    odd = torch.empty(3 * V + 1, device="cuda")
    odd[1:] = x.view(-1)
    again = call(ctx, 1, 3, odd[1:], tokens, 1.0, 3)
    assert all(torch.equal(a, b) for a, b in zip(again, (lp, ent, ids, top)))
    one = call(ctx, 1, 1, x[1].contiguous(), tokens[1:], 1.0, 3)
    assert torch.equal(one[0][0, 0], lp[0, 1]) and torch.equal(one[1][0, 0], ent[0, 1]) and torch.equal(one[3][0, 0], top[0, 1])
    ctx.close()


def test_refusals():
    ctx = context(batch=2, q=3, vocab=20)
    x, tokens = logits(6, 20, 7)
    f, i = torch.empty(400, device="cuda"), torch.empty(400, dtype=torch.int32, device="cuda")

    def code(*a):
        with pytest.raises(B.SdsatError) as e:
            B.sdsat_token_logprobs(ctx.handle, *a)
        return e.value.code
    assert code(3, 3, x, tokens, 1.0, 0, f, f, None, None) == -4
    assert code(2, 4, x, tokens, 1.0, 0, f, f, None, None) == -4
    assert code(0, 3, x, tokens, 1.0, 0, f, f, None, None) == -1
    assert code(2, 3, None, tokens, 1.0, 0, f, f, None, None) == -1
    assert code(2, 3, x, None, 1.0, 0, f, f, None, None) == -1
    for T in (0.0, -1.0, math.nan, math.inf, 1e-39):
        assert code(2, 3, x, tokens, T, 0, f, f, None, None) == -1
    assert code(2, 3, x, tokens, 1.0, -1, f, f, i, f) == -1
    assert code(2, 3, x, tokens, 1.0, 33, f, f, i, f) == -1
    assert code(2, 3, x, tokens, 1.0, 21, f, f, i, f) == -1        # more than there are ids
    assert code(2, 3, x, tokens, 1.0, 2, f, f, None, f) == -1
    assert code(2, 3, x, tokens, 1.0, 2, f, f, i, None) == -1
    ctx.close()


def test_captured_on_a_stream_of_its_own():
    V = 32016
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = context(batch=2, q=3, vocab=V)
        x, tokens = logits(6, V, 8)
        out = [torch.empty((2, 3), device="cuda"), torch.empty((2, 3), device="cuda"),
               torch.empty((2, 3, 5), dtype=torch.int32, device="cuda"), torch.empty((2, 3, 5), device="cuda")]
        s.synchronize()
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        for graph in graphs:   # two graphs that share the context's workspace, replayed one after the other
            with torch.cuda.graph(graph, stream=s):
                B.sdsat_token_logprobs(ctx.handle, 2, 3, x, tokens, 1.0, 5, *out)
        for i in range(6):
            x.copy_(logits(6, V, 20 + i)[0])
            for t in out:
                t.fill_(-7)
            graphs[i % 2].replay()
            s.synchronize()
            check(x, tokens, 1.0, 5, out)
            again = call(ctx, 2, 3, x, tokens, 1.0, 5)
            assert all(torch.equal(a, b) for a, b in zip(again, out))
    ctx.close()
