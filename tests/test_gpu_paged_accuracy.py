"""How far attention over a bf16 pool is from its definition in 64 bits: the weights are no rounding point but where long
chunks' outputs are rounded to bf16 themselves."""
import math

import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import paged_helpers   # noqa: E402
from paged_helpers import Call, assert_within, int64, tree_mask   # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def fine(monkeypatch):
    """Weights of 16 bits: half a step of bf16 left by the value, of which half a step of bf16 is left by the remainder."""
    monkeypatch.setitem(paged_helpers.HALF_STEP, torch.bfloat16, 2.0 ** -16)


HEADS = [(4, 4, 128), (8, 2, 64), (7, 1, 128), (40, 8, 128)]
SHORT = [[(1, 0), (1, 31), (1, 700)], [(6, 90), (1, 2000), (3, 0)], [(8, 333), (0, 5), (2, 1500)]]


@pytest.mark.parametrize("heads,kv,dh", HEADS)
@pytest.mark.parametrize("seqs", SHORT, ids=lambda s: "_".join(f"{n}at{c}" for n, c in s))
@pytest.mark.parametrize("out", ["bf16", "fp32"])
def test_short_chunks(monkeypatch, heads, kv, dh, seqs, out):
    print(f"case {heads}/{kv}x{dh} {seqs} {out}", flush=True)
    c = Call(seqs, heads, kv, dh, seed=1)
    q = c.randn((c.rows, heads * dh), scale=2.0)
    got = c.attend(q, out=torch.zeros_like(q, dtype=paged_helpers.TYPES[out]))
    fine(monkeypatch)
    assert_within(got, *c.expected(q, u_out=2.0 ** -8 if out == "bf16" else 2.0 ** -24))


@pytest.mark.parametrize("heads,kv,dh", HEADS)
def test_trees_and_windows(monkeypatch, heads, kv, dh):
    print(f"case {heads}/{kv}x{dh}", flush=True)
    c = Call([(9, 77), (9, 0), (9, 1300)], heads, kv, dh, seed=2)
    q = c.randn((c.rows, heads * dh), scale=2.0)
    mask = int64(tree_mask(9) * 3)
    float_out = lambda: torch.zeros_like(q, dtype=torch.float32)
    tree, windowed = c.attend(q, mask=mask, out=float_out()), c.attend(q, window=100, out=float_out())
    fine(monkeypatch)
    assert_within(tree, *c.expected(q, mask=mask, u_out=2.0 ** -24))
    assert_within(windowed, *c.expected(q, window=100, u_out=2.0 ** -24))


@pytest.mark.parametrize("heads,kv,dh", HEADS)
@pytest.mark.parametrize("window", [0, 150])
def test_long_chunks_with_float_outputs(monkeypatch, heads, kv, dh, window):
    print(f"case {heads}/{kv}x{dh} window {window}", flush=True)
    c = Call([(130, 0), (1, 400), (200, 777), (70, 31)], heads, kv, dh, seed=3)
    q = c.randn((c.rows, heads * dh), scale=2.0)
    got = c.attend(q, window=window, out=torch.zeros_like(q, dtype=torch.float32))
    rounded = c.attend(q, window=window)
    assert_within(rounded, *c.expected(q, window=window))
    fine(monkeypatch)
    assert_within(got, *c.expected(q, window=window, u_out=2.0 ** -24))


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("n", [1, 6, 90])
@pytest.mark.parametrize("at", [3, 95])
def test_values_that_are_not_finite_meet_no_remainder(n, at, value):
    """An infinity in a slot that every row sees, in a whole page and in one that ends at the chunk: it reaches its column,
    with its sign, and no other."""
    print(f"case n {n} slot {at} {value}", flush=True)
    c = Call([(n, 96)], 4, 2, 64, seed=4)
    q = c.randn((c.rows, 256))
    want, tol = c.expected(q)
    page, place = int(c.pages[0, at // 32]), paged_helpers.place(at)
    c.v[page, 0, 5, place] = value
    for out_type in (torch.bfloat16, torch.float32):
        got = c.attend(q, out=torch.zeros_like(q, dtype=out_type)).view(n, 4, 64)
        column = got[:, :2, 5]
        assert column.isnan().all() if math.isnan(value) else (column == value).all()
        rest = torch.ones(4, 64, dtype=torch.bool, device="cuda")
        rest[:2, 5] = False
        assert_within(got[:, rest], want.view(n, 4, 64)[:, rest], tol.view(n, 4, 64)[:, rest])
