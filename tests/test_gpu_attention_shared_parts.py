"""Shared-prefix attention beyond short caches and small trees: own slots cut into several parts, ancestor masks of up to
64 rows."""
import pytest
import torch

import helpers
from operator_helpers import device_error
from paper_2403_18647_amd import binding as B
from paper_2403_18647_amd import synth
from test_gpu_attention_shared import case, chain, check, reference, run

pytestmark = pytest.mark.gpu

MODELS = [("bf16", 2, 128), ("bf16", 3, 64), ("fp32", 2, 64), ("fp32", 1, 128)]
PART = 1024   # slots of an own part where the capacity is a few of them: it begins at the sequence's first own page


def own_lengths(group, prefix, lengths):
    """Committed slots behind the prefix, for lengths counted from the sequence's first own page."""
    return [p // 32 * 32 + n - p for p, n in zip([p for p in prefix for _ in range(group)], lengths)]


@pytest.mark.parametrize("dtype,heads,dh", MODELS)
@pytest.mark.parametrize("q", [1, 6, 40])
@pytest.mark.parametrize("lengths", [
    lambda q: [PART - 1, PART, PART + 1, 2 * PART + 100],          # committed slots end around the first border
    lambda q: [PART - q, PART - q + 1, 30, 2 * PART - q],          # the block ends at a border, a row past it, far before
    lambda q: [PART - q - 1, 2 * PART, 2 * PART - 1, 2 * PART + 1]])
def test_own_slots_in_several_parts(dtype, heads, dh, q, lengths):
    group, prefix = 2, [70, 500]
    own = own_lengths(group, prefix, lengths(q))
    ctx, keys, vals, x = case(dtype, heads, dh, group, prefix, own, q, slots=500 + 2 * PART + 200, seed=q)
    ref, tol = reference(keys, vals, x, q, chain(keys, q))
    check(run(ctx, group, prefix, q, x), ref, tol)
    assert device_error(ctx) == 0
    ctx.close()


@pytest.mark.parametrize("group,q", [(2, 6), (4, 11), (3, 1)])
def test_own_slots_in_several_parts_of_model_heads(group, q):
    """Heads of the 7B decoder with few sequences, whose own slots are far longer than their prefix."""
    prefix = [333]
    own = [3000 - 211 * b for b in range(group)]
    ctx, keys, vals, x = case("bf16", 32, 128, group, prefix, own, q, slots=3400, seed=q)
    ref, tol = reference(keys, vals, x, q, chain(keys, q))
    check(run(ctx, group, prefix, q, x), ref, tol)
    ctx.close()


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("fp32", 64)])
@pytest.mark.parametrize("border", [PART, 2 * PART])
def test_a_row_does_not_depend_on_its_block_across_parts(dtype, dh, border):
    """A block whose rows lie on both sides of a part's end: each is bitwise the row of any shorter block."""
    q, group, prefix = 40, 2, 70
    own = own_lengths(group, [prefix], [border - 18, border - 13])
    ctx, keys, vals, x = case(dtype, 2, dh, group, [prefix], own, q, slots=prefix + 2 * PART + 200)
    whole = run(ctx, group, [prefix], q, x).view(group, q, -1)
    ref, tol = reference(keys, vals, x, q, chain(keys, q))
    check(whole.reshape(group * q, -1), ref, tol)
    for rows in (1, 5, 17):
        for r in (0, 12, 13, 17, 18, 23):
            B.sdsat_set_cache_len(ctx.handle, [prefix + n + r for n in own])
            part = x.view(group, q, -1)[:, r:r + rows].contiguous().view(group * rows, -1)
            got = run(ctx, group, [prefix], rows, part).view(group, rows, -1)
            assert torch.equal(got, whole[:, r:r + rows]), (rows, r)
    ctx.close()


@pytest.mark.parametrize("dtype,dh,q", [("bf16", 128, 3), ("fp32", 64, 3), ("bf16", 64, 40)])
def test_replays_and_eager_calls_agree_with_the_reference(dtype, dh, q):
    """A graph captured while the sequences were short puts all own slots into one part, an eager call several."""
    prefix, own = [70], [2100, 1500]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx, keys, vals, x = case(dtype, 2, dh, 2, prefix, own, q, slots=4000)
        out = torch.full_like(x, 7e7)
        B.sdsat_set_cache_len(ctx.handle, [75, 71])
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.sdsat_attention_shared(ctx.handle, 0, 2, q, 2, prefix, x, None, out)
        B.sdsat_set_cache_len(ctx.handle, [prefix[0] + n for n in own])
        ref, tol = reference(keys, vals, x, q, chain(keys, q))
        for _ in range(3):
            out.fill_(7e7)
            graph.replay()
            s.synchronize()
            check(out, ref, tol)
            check(run(ctx, 2, prefix, q, x), ref, tol)
        assert device_error(ctx) == 0
    ctx.close()


def random_masks(n, q, seed, empty):
    """[n, q, q] truth values: any row may see any other, some see none; and the same as 64-bit masks."""
    g = torch.Generator().manual_seed(seed)
    see = torch.rand((n, q, q), generator=g) < 0.3
    see[:, torch.arange(q), torch.arange(q)] = True
    for r in empty:
        see[(r // 3) % n, r] = False
    words = [sum(1 << j for j in range(q) if row[j]) for row in see.view(n * q, q).tolist()]
    words = [w - (1 << 64) if w >> 63 else w for w in words]
    return see.cuda(), torch.tensor(words, dtype=torch.int64, device="cuda")


@pytest.mark.parametrize("dtype,heads,dh", MODELS)
@pytest.mark.parametrize("q", [16, 17, 33, 48, 64])
@pytest.mark.parametrize("prefix,own", [([40, 0], [3, 20, 0, 31]),         # blocks across two and three pages
                                        ([0, 31], [0, 0, 1, 0]),
                                        ([64, 96], [PART - 40, 0, PART - 1, 5])])
def test_masks_of_many_rows(dtype, heads, dh, q, prefix, own):
    """Every row tile of a block, mask bits from 32 up, other masks for each sequence, rows that see no row."""
    empty = [r for r in (0, 3, 15, 16, 18, 32, 34, 47, 48, 63) if r < q]
    see, mask = random_masks(4, q, q, empty)
    ctx, keys, vals, x = case(dtype, heads, dh, 2, prefix, own, q, slots=max(prefix) + max(own) + q + 900, seed=q)
    sees = [torch.cat([torch.ones((q, k.shape[1] - q), dtype=torch.bool, device="cuda"), see[b]], 1)
            for b, k in enumerate(keys)]
    ref, tol = reference(keys, vals, x, q, sees)
    out = run(ctx, 2, prefix, q, x, mask)
    check(out, ref, tol)
    for b, s in enumerate(sees):
        for r in range(q):
            assert bool(s[r].any()) or not bool(out[b * q + r].any())
    ctx.close()


@pytest.mark.parametrize("name", ["tiny", "small"])
@pytest.mark.parametrize("q", [20, 32])
def test_tree_blocks_of_many_rows(name, q):
    """Whole forward blocks with trees of more than one row tile, against sequences that hold the prefix themselves."""
    wl = synth.workload("tiny") if name == "tiny" else helpers.small_bf16()
    sh, n, P = wl.shape, 2, 75
    tol = 1e-4 if sh.dtype == "fp32" else 3e-2   # the framework's bounds for logits of two-layer models
    prompt = torch.from_numpy(synth.prompts(wl, 1, P)[0].astype("int32")).cuda()
    parent = [-1] + [max(0, r - 1 - r % 5) for r in range(1, q)]
    words = []
    for r in range(q):
        words.append((words[parent[r]] if r else 0) | 1 << r)
    mask = torch.tensor(words * n, dtype=torch.int64, device="cuda")
    t = torch.randint(0, sh.vocab, (n, q), generator=torch.Generator().manual_seed(q), dtype=torch.int32).cuda()
    got = []
    for first in (P, 0):
        ctx = helpers.make_ctx(wl, n, 200, P)
        B.sdsat_forward_block(ctx.handle, 1, P, prompt, None, None)
        B.sdsat_commit_kv(ctx.handle, 1, P, torch.tensor([P], dtype=torch.int32, device="cuda"))
        B.sdsat_kv_reorder(ctx.handle, n, torch.zeros(n, dtype=torch.int32, device="cuda"), first)
        lg = torch.empty((n * q, sh.vocab), device="cuda")
        if first:
            B.sdsat_forward_block_shared(ctx.handle, n, q, n, [P], t, mask, lg)
        else:
            B.sdsat_forward_block(ctx.handle, n, q, t, mask, lg)
        torch.cuda.synchronize()
        got.append(lg)
        assert device_error(ctx) == 0
        ctx.close()
    assert float((got[0] - got[1]).abs().max()) <= tol
