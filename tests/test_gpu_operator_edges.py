"""Calls at the ends of what cache reordering, shared-prefix attention and token log probabilities take: outputs in place of
the queries, the most groups, sequences around a wave's lanes and the most of them, as many alternatives as ids, two contexts at work
at once."""
import random

import pytest
import torch

from operator_helpers import context, device_error
from paper_2403_18647_amd import binding as B
from test_gpu_attention_shared import case, chain, check, reference, run
from test_gpu_kv_reorder import check as check_reorder
from test_gpu_token_logprobs import call, logits
from test_gpu_token_logprobs import check as check_logprobs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("fp32", 64)])
@pytest.mark.parametrize("q", [1, 6, 40, 70, 130])
@pytest.mark.parametrize("group", [1, 2, 4])
def test_outputs_in_place_of_the_queries(dtype, dh, q, group):
    prefix = [100] * (4 // group)
    ctx, keys, vals, x = case(dtype, 3, dh, group, prefix, [5, 40, 0, 33], q)
    want = run(ctx, group, prefix, q, x)
    for _ in range(3):
        there = x.clone()
        B.sdsat_attention_shared(ctx.handle, 0, 4, q, group, prefix, there, None, there)
        torch.cuda.synchronize()
        assert torch.equal(there, want)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("q", [1, 9])
def test_the_most_groups(dtype, q):
    prefix = [(37 * i) % 200 for i in range(64)]
    own = [(11 * b) % 50 for b in range(128)]
    ctx, keys, vals, x = case(dtype, 1, 64, 2, prefix, own, q)
    ref, tol = reference(keys, vals, x, q, chain(keys, q))
    check(run(ctx, 2, prefix, q, x), ref, tol)
    assert device_error(ctx) == 0
    ctx.close()
    big = context(1, 64, dtype, 1, 130, 64, 1)
    x = torch.zeros((130, 64), device="cuda")
    for group in (1, 2):
        with pytest.raises(B.SdsatError) as e:
            B.sdsat_attention_shared(big.handle, 0, 65 * group, 1, group, [0] * 65, x, None, x)
        assert e.value.code == -5
    big.close()


def test_one_large_group():
    """130 sequences of one prefix: as many rows as the largest prefill tile three times over."""
    prefix, own, q = [300], [b % 40 for b in range(130)], 2
    ctx, keys, vals, x = case("bf16", 2, 64, 130, prefix, own, q)
    ref, tol = reference(keys, vals, x, q, chain(keys, q))
    check(run(ctx, 130, prefix, q, x), ref, tol)
    ctx.close()


@pytest.mark.parametrize("n", [63, 64, 65, 1024])
def test_sequences_around_a_wave_s_lanes_and_the_most(n):
    rng = random.Random(n)
    ctx = context(1, 64, "bf16", batch=n, slots=64)
    around = [(b + 1) % n for b in range(n)]
    pairs = [b ^ 1 if b ^ 1 < n else b for b in range(n)]
    shuffled = list(range(n))
    rng.shuffle(shuffled)
    for i, src in enumerate((around, pairs, shuffled, [n - 1] * n, [max(0, b - 1) for b in range(n)],
                             [rng.randint(-1, n - 1) for _ in range(n)], [rng.randint(0, 3) for _ in range(n)],
                             shuffled[:n - 1])):
        check_reorder(ctx, [rng.randint(0, 64) for _ in range(n)], src, 32 * (i % 2), seed=i)
    assert device_error(ctx) == 0
    ctx.close()


def test_more_sequences_than_a_reordering_takes():
    ctx = context(1, 64, "bf16", batch=1025, slots=32)
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_kv_reorder(ctx.handle, 4, torch.zeros(4, dtype=torch.int32, device="cuda"), 0)
    assert e.value.code == -5
    ctx.close()


@pytest.mark.parametrize("V", [2, 3, 32])
def test_as_many_alternatives_as_ids(V):
    ctx = context(batch=2, q=2, vocab=V)
    x, tokens = logits(4, V, V)
    check_logprobs(x, tokens, 1.0, V, call(ctx, 2, 2, x, tokens, 1.0, V))
    ctx.close()


def test_two_contexts_at_work_at_once():
    """Each on a stream of its own, with their own caches and scratch."""
    q, prefix, V = 6, [200], 9000
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = []
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            ctx, keys, vals, x = case("bf16", 4, 128, 4, prefix, [5, 60, 0, 31], q, seed=i)
            lctx = context(batch=4, q=q, vocab=V)
            z, tokens = logits(4 * q, V, i)
            s.synchronize()
            want = run(ctx, 4, prefix, q, x), call(lctx, 4, q, z, tokens, 1.0, 5)
            work.append((ctx, lctx, x, z, tokens, want))
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for s, (ctx, lctx, x, z, tokens, _w) in zip(streams, work):
            with torch.cuda.stream(s):
                out = torch.empty_like(x)
                lp, ent = torch.empty((4, q), device="cuda"), torch.empty((4, q), device="cuda")
                ids, top = torch.empty((4, q, 5), dtype=torch.int32, device="cuda"), torch.empty((4, q, 5), device="cuda")
                B.sdsat_attention_shared(ctx.handle, 0, 4, q, 4, prefix, x, None, out)
                B.sdsat_token_logprobs(lctx.handle, 4, q, z, tokens, 1.0, 5, lp, ent, ids, top)
                outs.append((out, (lp, ent, ids, top)))
    torch.cuda.synchronize()
    for i, (out, lps) in enumerate(outs):
        want = work[i % 2][5]
        assert torch.equal(out, want[0]) and all(torch.equal(a, b) for a, b in zip(lps, want[1]))
    for w in work:
        w[0].close()
        w[1].close()
