"""The parts of shared-prefix attention lie over scratch of the other calls: each call gives what it gives on a context that
makes no other, in any order, eagerly and replayed."""
import numpy as np
import pytest
import torch

import helpers
from paper_2403_18647_amd import binding as B
from paper_2403_18647_amd import synth

pytestmark = pytest.mark.gpu

P, N = 77, 4


def prepared(wl, prompt, batch=N):
    """A context whose sequences hold the prompt's first P tokens, all but the first in their own last page only."""
    ctx = helpers.make_ctx(wl, batch, 400, 90)
    fill(ctx, prompt)
    return ctx


def fill(ctx, prompt):
    B.sdsat_reset(ctx.handle, N)
    t = torch.from_numpy(np.ascontiguousarray(prompt[:P], np.int32)).cuda()
    B.sdsat_forward_block(ctx.handle, 1, P, t, None, None)
    B.sdsat_commit_kv(ctx.handle, 1, P, torch.tensor([P], dtype=torch.int32, device="cuda"))
    B.sdsat_kv_reorder(ctx.handle, N, torch.zeros(N, dtype=torch.int32, device="cuda"), 0)


@pytest.mark.parametrize("name", ["tiny", "small"])
def test_calls_in_any_order(name):
    wl = synth.workload("tiny") if name == "tiny" else helpers.small_bf16()
    sh, k = wl.shape, wl.k
    prompt = synth.prompts(wl, 1, P + 1)[0]
    ad = synth.adaptive_ids(sh, k)
    g = torch.Generator().manual_seed(9)
    tokens = {q: torch.randint(0, sh.vocab, (N, q), generator=g, dtype=torch.int32).cuda() for q in (3, 16, 40, 90)}

    def block(ctx, q, group):
        lg = torch.empty((N * q, sh.vocab), device="cuda")
        if group:
            B.sdsat_forward_block_shared(ctx.handle, N, q, group, [P] * (N // group), tokens[q], None, lg)
        else:
            B.sdsat_forward_block(ctx.handle, N, q, tokens[q], None, lg)
        torch.cuda.synchronize()
        return lg

    def attention(ctx, q, group):
        r = torch.Generator().manual_seed(q)
        x, kn, vn = (torch.randn((N * q, sh.d_model), generator=r).cuda() for _ in range(3))
        pos = torch.arange(P, P + q, dtype=torch.int32, device="cuda").repeat(N)
        B.sdsat_kv_write(ctx.handle, 1, N, q, kn, vn, pos)   # the block's own rows
        out = torch.empty_like(x)
        B.sdsat_attention_shared(ctx.handle, 1, N, q, group, [P] * (N // group), x, None, out)
        torch.cuda.synchronize()
        return out

    def generate(ctx):
        out, _ = B.sdsat_generate(ctx.handle, np.stack([prompt[:20]] * 2), 24, k, ad)
        fill(ctx, prompt)
        return torch.from_numpy(np.asarray(out))

    calls = {"generate": generate}
    for q in tokens:
        for group in (0, 2, 4):
            calls[f"block {q} {group}"] = lambda c, q=q, group=group: block(c, q, group)
            if group:
                calls[f"attention {q} {group}"] = lambda c, q=q, group=group: attention(c, q, group)
    want = {}
    for what, f in calls.items():   # each on a context of its own
        ctx = prepared(wl, prompt)
        want[what] = f(ctx)
        ctx.close()
    ctx = prepared(wl, prompt)
    order = list(calls) * 3
    np.random.default_rng(4).shuffle(order)
    for what in order:
        assert torch.equal(calls[what](ctx), want[what]), what
    ctx.close()


@pytest.mark.parametrize("name", ["tiny", "small"])
@pytest.mark.parametrize("q", [5, 40])
def test_replayed_between_other_calls(name, q):
    """Graphs of a shared and of a plain block, replayed in turn with eager calls between them."""
    wl = synth.workload("tiny") if name == "tiny" else helpers.small_bf16()
    sh = wl.shape
    prompt = synth.prompts(wl, 1, P + 1)[0]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = prepared(wl, prompt)
        t = torch.randint(0, sh.vocab, (N, q), generator=torch.Generator().manual_seed(q), dtype=torch.int32).cuda()
        shared, plain, other = (torch.empty((N * q, sh.vocab), device="cuda") for _ in range(3))
        s.synchronize()
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        with torch.cuda.graph(graphs[0], stream=s):
            B.sdsat_forward_block_shared(ctx.handle, N, q, 4, [P], t, None, shared)
        with torch.cuda.graph(graphs[1], stream=s):
            B.sdsat_forward_block(ctx.handle, N, q, t, None, plain)
        for i in range(5):
            t.copy_(torch.randint(0, sh.vocab, (N, q), generator=torch.Generator().manual_seed(50 + i), dtype=torch.int32).cuda())
            for g in graphs if i % 2 else graphs[::-1]:
                g.replay()
            s.synchronize()
            B.sdsat_forward_block_shared(ctx.handle, N, q, 4, [P], t, None, other)
            s.synchronize()
            assert torch.equal(shared, other)
            B.sdsat_forward_block(ctx.handle, N, q, t, None, other)
            s.synchronize()
            assert torch.equal(plain, other)
            shared.fill_(7e7)
            plain.fill_(7e7)
    ctx.close()
