"""What calls on a paged cache say of numbers that do not fit, where nothing else is left to compute or rows overlap."""
import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paged_helpers import Call, assert_within   # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def assert_reported(c, code=-6):
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_paged_status(c.handle)
    assert e.value.code == code
    B.sdsat_paged_status(c.handle)   # once


@pytest.mark.parametrize("count", [3, 9, 70])
@pytest.mark.parametrize("n", [6, 200])
def test_starts_that_go_back_and_forth(n, count):
    """Several sequences with the same rows, more tiles than the rows make: reported, and the next call is right."""
    print(f"case {count} sequences of {n}", flush=True)
    c = Call([(n, 40)] * count, 4, 2, 64)
    q = c.randn((c.rows, 256))
    want, tol = c.expected(q)
    good, rows = c.d_start.clone(), c.rows
    c.d_start.copy_(torch.tensor([n * (i % 2) for i in range(count + 1)], dtype=torch.int32))
    c.rows = n
    c.batch = B.paged_batch(c.d_start, c.d_len, c.pages, n, n, n + 40)
    out = torch.full_like(q, 3.0)
    c.attend(q, out=out)
    assert_reported(c)
    assert (out[n:] == 3).all()
    c.d_start.copy_(good)
    c.rows = rows
    c.batch = B.paged_batch(c.d_start, c.d_len, c.pages, rows, n, n + 40)
    assert_within(c.attend(q), want, tol)
    B.sdsat_paged_status(c.handle)
