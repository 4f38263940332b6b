"""Rules on logits against their definition."""
import math

import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from operator_helpers import context, device_error   # noqa: E402
from paged_helpers import int64, tree_mask   # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def expected(batch, q, vocab, logits, r):
    """In 64 bits; and the size of what was added, for the roundings."""
    z = logits.double().view(batch, q, vocab).clone()
    size = z.abs()
    for b in range(batch):
        old = said0 = torch.zeros(vocab, dtype=torch.int64, device="cuda")
        if r.get("history") is not None:
            n = int(r["history_len"][b])
            prompt = int(r["prompt_len"][b]) if r.get("prompt_len") is not None else 0
            h = r["history"][b, :n].long()
            ok = (h >= 0) & (h < vocab)
            i = torch.arange(n, device="cuda")
            old = torch.bincount(h[ok & (i < prompt)], minlength=vocab)
            said0 = torch.bincount(h[ok & (i >= prompt)], minlength=vocab)
        for j in range(q):
            said = said0.clone()
            if r.get("tokens") is not None:
                bits = int(r["mask"][b * q + j]) if r.get("mask") is not None else (2 << j) - 1
                for i in range(q):
                    t = int(r["tokens"][b, i])
                    if bits >> i & 1 and 0 <= t < vocab:
                        said[t] += 1
            row = z[b, j]
            rep, freq, pres = (float(x) for x in r["penalties"][:, b]) if r.get("penalties") is not None else (1.0, 0.0, 0.0)
            row = torch.where(said + old > 0, torch.where(row > 0, row / rep, row * rep), row)
            row = row - freq * said - pres * (said > 0)
            size[b, j] = row.abs().nan_to_num(0, 0, 0) + 2 * abs(freq) * said + 2 * abs(pres) * (said > 0)
            if r.get("bias") is not None:
                bias = r["bias"].view(-1, vocab)[b if r["bias"].numel() > vocab else 0].double()
                row = row + bias
                size[b, j] += bias.abs().nan_to_num(0, 0, 0)
            if r.get("allowed") is not None:
                ids = torch.arange(vocab, device="cuda")
                row = torch.where((r["allowed"][b * q + j][ids // 32] >> (ids % 32) & 1) == 1, row, -math.inf)
            z[b, j] = row
    return z.view(batch * q, vocab), size.view(batch * q, vocab)


def check(batch, q, vocab, r, logits, in_place=False):
    c = context(batch=batch, q=max(q, 1), vocab=vocab)
    want, size = expected(batch, q, vocab, logits, r)
    given = logits.clone()
    out = given if in_place else torch.full_like(logits, 7.0)
    B.sdsat_adjust_logits(c.handle, batch, q, given, B.logit_rules(**r), out)
    assert device_error(c) == 0
    assert in_place or torch.equal(given.view(torch.int32), logits.view(torch.int32))
    # six float operations; what lies past float's range (-3.4e38 times a penalty of 1.3) rounds to infinity
    same = (out == want.float()) | (out.isnan() & want.isnan())
    off = (out.double() - want).abs()
    assert (same | (off <= 6 * 2.0 ** -24 * 1.01 * size)).all(), float((off - 6 * 2.0 ** -24 * size).nan_to_num(0).max())
    c.close()
    return out


def rules(g, batch, q, vocab, hist, tree=0, grammar=True, bias="each", words=None):
    words = words or max(1, vocab // 20)
    r = {}
    if hist:
        r["history"] = torch.randint(-2, words + 3, (batch, hist), generator=g, device="cuda").int()
        r["history"][:, ::13] = vocab + 5
        r["history_len"] = torch.randint(0, hist + 1, (batch,), generator=g, device="cuda").int()
        r["history_len"][0] = hist
        r["prompt_len"] = (r["history_len"] * 0.4).int()
    if q <= 64:
        r["tokens"] = torch.randint(0, words, (batch, q), generator=g, device="cuda").int()
        r["tokens"][:, -1] = vocab + 1   # an adaptive token
        if tree:
            r["mask"] = int64((tree_mask(q, tree) + [5] * q)[:q] * batch)
    r["penalties"] = torch.stack([0.8 + torch.rand(batch, generator=g, device="cuda"),
                                  torch.randn(batch, generator=g, device="cuda"),
                                  torch.randn(batch, generator=g, device="cuda")])
    if bias:
        r["bias"] = torch.randn((1 if bias == "shared" else batch, vocab), generator=g, device="cuda")
        r["bias"][:, ::17] = -math.inf
    if grammar:
        r["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (batch * q, (vocab + 31) // 32), generator=g, device="cuda").int()
    return r


def gen(seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("batch,q,vocab,hist,tree,grammar,bias", [
    (1, 1, 2, 3, 0, True, "shared"), (1, 6, 1000, 800, 0, False, None), (3, 5, 1024, 1, 2, True, "each"),
    (2, 11, 1025, 4097, 2, True, "shared"), (4, 7, 32017, 333, 0, True, "each"), (2, 64, 2047, 100, 2, True, "each"),
    (1, 3, 50257, 9000, 0, False, "shared"), (2, 6, 128256, 2000, 0, True, "shared"), (1, 90, 4001, 50, 0, True, "each"),
    (5, 2, 31, 7, 0, True, None)])
def test_against_definition(batch, q, vocab, hist, tree, grammar, bias):
    print(f"case {batch}x{q}x{vocab} history {hist}", flush=True)
    g = gen(q)
    r = rules(g, batch, q, vocab, hist, tree, grammar, bias)
    logits = torch.randn((batch * q, vocab), generator=g, device="cuda") * 4
    check(batch, q, vocab, r, logits)
    check(batch, q, vocab, r, logits, in_place=True)


@pytest.mark.parametrize("leave", ["history", "tokens", "prompt_len", "mask", "penalties", "bias", "allowed", "all", "history_tokens"])
def test_any_rule_may_be_left_out(leave):
    batch, q, vocab = 3, 5, 1111
    r = rules(gen(1), batch, q, vocab, 200, 2)
    if leave == "all":
        r = {}
    for name in leave.split("_") if leave == "history_tokens" else [leave]:
        r.pop(name, None)
    if "history" not in r:
        r.pop("history_len", None), r.pop("prompt_len", None)
    if "tokens" not in r:
        r.pop("mask", None)
    logits = torch.randn((batch * q, vocab), generator=gen(2), device="cuda")
    out = check(batch, q, vocab, r, logits)
    assert leave != "all" or torch.equal(out, logits)


def test_special_logits_and_rows_without_ids():
    """NaN, infinities, zeros and the type's lowest value, seen and unseen; a row whose ids are all taken."""
    vocab = 1030
    z = torch.tensor([0.0, -0.0, math.nan, math.inf, -math.inf, -3.4028234663852886e38, 3.4028234663852886e38, 1e-45, 5.0, -5.0],
                     device="cuda").repeat(2 * 103).view(2, vocab).contiguous()
    r = {"history": torch.arange(500, dtype=torch.int32, device="cuda")[None].contiguous(),
         "history_len": torch.tensor([500], dtype=torch.int32, device="cuda"),
         "penalties": torch.tensor([[1.3], [0.5], [0.25]], device="cuda"),
         "allowed": torch.stack([torch.full((33,), -1), torch.zeros(33)]).int().cuda()}
    out = check(1, 2, vocab, r, z)
    assert (out[1] == -math.inf).all()


def test_counts_are_exact():
    """A token said 70000 times, all tokens of a block alike, and blocks whose rows see different ones."""
    vocab, n = 64, 70000
    r = {"history": torch.full((1, n), 5, dtype=torch.int32, device="cuda"),
         "history_len": torch.tensor([n], dtype=torch.int32, device="cuda"),
         "prompt_len": torch.tensor([1], dtype=torch.int32, device="cuda"),
         "tokens": torch.full((1, 64), 5, dtype=torch.int32, device="cuda"),
         "penalties": torch.tensor([[1.0], [1.0], [0.0]], device="cuda")}
    out = check(1, 64, vocab, r, torch.zeros((64, vocab), device="cuda"))
    assert torch.equal(out[:, 5], -torch.arange(n, n + 64, device="cuda").float())
    r["mask"] = int64([(1 << 64) - 1 - (1 << i) for i in range(64)])
    out = check(1, 64, vocab, r, torch.zeros((64, vocab), device="cuda"))
    assert (out[:, 5] == -(n - 1 + 63)).all()


def test_history_lengths_past_the_rows_are_reported():
    c = context(batch=2, q=1, vocab=64)
    z = torch.zeros((2, 64), device="cuda")
    for bad in (-1, 9, 2 ** 31 - 1):
        r = B.logit_rules(history=torch.zeros((2, 8), dtype=torch.int32, device="cuda"),
                          history_len=torch.tensor([3, bad], dtype=torch.int32, device="cuda"))
        B.sdsat_adjust_logits(c.handle, 2, 1, z, r, z.clone())
        assert device_error(c) == -6
        assert device_error(c) == 0


def test_rows_past_4_gib():
    """700 rows past 2^32 bytes into the logits."""
    batch, q, vocab = 16, 600, 131071
    c = context(batch=batch, q=q, vocab=vocab)
    z = torch.zeros((batch * q, vocab), device="cuda")
    z[-1] = torch.randn(vocab, generator=gen(), device="cuda")
    hist = torch.zeros((batch, 4), dtype=torch.int32, device="cuda")
    hist[-1] = torch.tensor([vocab - 1, 7, vocab - 1, vocab], dtype=torch.int32)
    pen = torch.tensor([[1.0], [0.5], [0.0]], device="cuda").repeat(1, batch)
    out = torch.full_like(z, 9.0)
    B.sdsat_adjust_logits(c.handle, batch, q, z, B.logit_rules(history=hist, history_len=torch.full((batch,), 4, dtype=torch.int32, device="cuda"),
                                                               penalties=pen), out)
    want = z[-1].clone()
    want[vocab - 1] -= 1.0
    want[7] -= 0.5
    assert torch.equal(out[-1], want)
    assert float(out[0, 0]) == -2.0 and (out[:, 1:7] == z[:, 1:7]).all()
