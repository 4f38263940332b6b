"""Prefixes of shared attention that are longer than a sequence: what the host and the device know of it."""
import pytest
import torch

from operator_helpers import context, device_error
from paper_2403_18647_amd import binding as B
from test_gpu_attention_shared import run

pytestmark = pytest.mark.gpu


def grown(slots, q, batch, length, commits):
    """A context whose sequences hold `length` slots while the host only knows a larger bound (commits of q rows)."""
    ctx = context(2, 64, "bf16", 1, batch, slots, q)
    for i in range(commits):
        rows = [n * (i + 1) // commits - n * i // commits for n in length]
        B.sdsat_commit_kv(ctx.handle, batch, q, torch.tensor(rows, dtype=torch.int32, device="cuda"))
    return ctx


@pytest.mark.parametrize("q", [3, 70])
@pytest.mark.parametrize("prefix,length,code", [
    ([70], [65, 70], -6), ([70], [70, 69], -6), ([70], [64, 200], -6), ([31], [0, 31], -6), ([1], [1, 0], -6),
    ([70], [70, 70], 0), ([31], [31, 31], 0), ([64], [64, 65], 0), ([0], [0, 0], 0),
    ([64, 33], [64, 64, 40, 32], -6), ([64, 33], [64, 64, 40, 33], 0)])
def test_prefixes_longer_than_a_sequence_by_less_than_a_page(prefix, length, code, q):
    n = len(length)
    ctx = grown(600, q, n, length, 200 // q + 6 if q < 70 else 5)
    x = torch.zeros((n * q, 128), device="cuda")
    run(ctx, 2, prefix, q, x)
    assert device_error(ctx) == code
    assert device_error(ctx) == 0
    ctx.close()


@pytest.mark.parametrize("group", [1, 2])
def test_lengths_that_the_capacity_check_reads_hold_for_the_prefix_too(group):
    """The bounds (90) say that a block may not fit: the true lengths (30) are read, and the prefix is compared with them."""
    ctx = grown(96, 9, 2, [30, 30], 10)
    x = torch.zeros((18, 128), device="cuda")
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_attention_shared(ctx.handle, 0, 2, 9, group, [31] * (2 // group), x, None, x.clone())
    assert e.value.code == -4
    t = torch.zeros((2, 9), dtype=torch.int32, device="cuda")
    ctx2 = grown(96, 9, 2, [30, 30], 10)
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_forward_block_shared(ctx2.handle, 2, 9, group, [31] * (2 // group), t, None, None)
    assert e.value.code == -4
    for c in (ctx, ctx2):
        B.sdsat_attention_shared(c.handle, 0, 2, 9, group, [30] * (2 // group), x, None, x.clone())
        assert device_error(c) == 0
        c.close()
