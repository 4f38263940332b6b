"""Rows of chunks of up to 64 packed rows over a paged cache: each one's bits, in its chunk and decoded alone."""
import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paged_helpers import Call, assert_within, place   # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


HEADS = [("bf16", 4, 4, 128), ("bf16", 8, 2, 64), ("bf16", 7, 1, 128), ("fp32", 2, 2, 64), ("fp32", 6, 2, 128)]


def alone(c, b, i, q, window=0, out_type=None):
    """Row i of sequence b of a call as a call of its own, on the same handle and pages."""
    row, slot = c.start[b] + i, c.seqs[b][1] + i
    t = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q[:1], dtype=out_type or q.dtype)
    B.sdsat_paged_attention(c.handle, B.paged_batch(t([0, 1]), t([slot]), c.pages[b:b + 1], 1, 1, slot + 1), c.k, c.v,
                            q[row:row + 1].contiguous(), None, window, 0.0, out)
    return out[0]


def assert_rows_alone(c, q, window=0, out_type=None):
    got = c.attend(q, window=window, out=torch.zeros_like(q, dtype=out_type or q.dtype))
    B.sdsat_paged_status(c.handle)
    for b, (n, _) in enumerate(c.seqs):
        assert n * (c.heads // c.kv) <= 64
        for i in range(n):
            same = torch.equal(got[c.start[b] + i], alone(c, b, i, q, window, out_type))
            assert same, f"row {i} of sequence {b}"
    return got


def climbing(c, top):
    """Keys that grow along the sequences, and queries of all sizes: each row's largest score moves at other pages."""
    for b, (n, cached) in enumerate(c.seqs):
        k, v = c.get(b, 0, n + cached)
        c.put(b, 0, k.float() * torch.linspace(0.1, top, n + cached, device="cuda")[:, None, None], v)
    size = 4 * torch.rand((c.rows, c.heads, 1), generator=c.g, device="cuda")
    return (c.randn((c.rows, c.heads, c.dh), torch.float32) * size).view(c.rows, -1).to(c.dtype)


@pytest.mark.parametrize("dtype,heads,kv,dh", HEADS)
@pytest.mark.parametrize("seed", range(3))
def test_rows_beside_rows_whose_scores_climb(dtype, heads, kv, dh, seed):
    """A row whose own maximum moves little keeps its bits beside rows whose maximum moves much."""
    most = 64 * kv // heads
    print(f"case {dtype} {heads}/{kv}x{dh} seed {seed}", flush=True)
    c = Call([(min(6, most), 700), (most, 95), (2, 2200)], heads, kv, dh, dtype, seed=seed)
    q = climbing(c, 2.0)
    got = assert_rows_alone(c, q)
    assert_within(got, *c.expected(q))


@pytest.mark.parametrize("dtype,heads,kv,dh", HEADS)
@pytest.mark.parametrize("window", [33, 90, 130])
def test_windows_that_begin_on_both_sides_of_a_page(dtype, heads, kv, dh, window):
    """The chunk's first rows see a page that its last ones do not."""
    print(f"case {dtype} {heads}/{kv}x{dh} window {window}", flush=True)
    c = Call([(6, 320 + window - 4), (8, 64 + window - 1), (7, 3 * window)], heads, kv, dh, dtype, seed=window)
    q = c.randn((c.rows, heads * dh), scale=2.0)
    got = assert_rows_alone(c, q, window)
    assert_within(got, *c.expected(q, window=window))


@pytest.mark.parametrize("dtype,heads,kv,dh", HEADS)
@pytest.mark.parametrize("window", [1400, 2900])
def test_windows_that_begin_on_both_sides_of_a_part(dtype, heads, kv, dh, window):
    """Parts are 512 slots of this handle; the chunk's first rows see one more of them than its last ones."""
    print(f"case {dtype} {heads}/{kv}x{dh} window {window}", flush=True)
    c = Call([(6, 512 * j + window - 4) for j in (1, 2, 3)] + [(8, 1024 + window - 8)], heads, kv, dh, dtype, max_ctx=6000, seed=window)
    q = c.randn((c.rows, heads * dh), scale=2.0)
    got = assert_rows_alone(c, q, window, torch.float32)
    assert_within(got, *c.expected(q, window=window, u_out=2.0 ** -24))


@pytest.mark.parametrize("dtype,heads,kv,dh", HEADS)
def test_masks_of_a_chain(dtype, heads, kv, dh):
    """Rows whose mask allows their own and the earlier ones, beside branches that see less: the bits of a single token."""
    most = 64 * kv // heads
    print(f"case {dtype} {heads}/{kv}x{dh}", flush=True)
    c = Call([(min(8, most), 1020), (most, 61), (min(5, most), 0)], heads, kv, dh, dtype, seed=11)
    q = climbing(c, 2.0)
    chain = torch.tensor([(2 << i) - 1 if i < 63 else -1 for n, _ in c.seqs for i in range(n)], dtype=torch.int64, device="cuda")
    mask = chain.clone()
    branch = torch.tensor([i for b, (n, _) in enumerate(c.seqs) for i in range(c.start[b], c.start[b] + n) if (i - c.start[b]) % 3 == 2],
                          device="cuda")
    mask[branch] &= 0x5555555555555555
    got = c.attend(q, mask=mask)
    assert_within(got, *c.expected(q, mask=mask))
    for b, (n, _) in enumerate(c.seqs):
        for i in range(n):
            if mask[c.start[b] + i] == chain[c.start[b] + i]:
                same = torch.equal(got[c.start[b] + i], alone(c, b, i, q))
                assert same, f"row {i} of sequence {b}"


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype,heads,kv,dh", HEADS)
def test_values_that_are_not_finite_with_weights_of_zero(dtype, heads, kv, dh, value):
    """A slot whose weight is below the smallest float and whose value is not finite makes NaN of the rows that see it, in a
    page that the chunk sees in part as in one that a single token sees whole; rows ahead of it do not meet it."""
    print(f"case {dtype} {heads}/{kv}x{dh} {value}", flush=True)
    n, cached, at = 6, 60, 61
    c = Call([(n, cached)], heads, kv, dh, dtype, seed=5)
    q = c.randn((c.rows, heads * dh)).abs() + 1
    page, slot = c.slots(0, at, at + 1)
    c.k[page, :, slot] = -40.0   # scores of -40 sqrt(dh) and less
    for out_type in (None, torch.float32):
        before = c.attend(q, out=torch.zeros_like(q, dtype=out_type or q.dtype))
        keep = c.v.clone()
        c.v[page, 0, 7, place(at)] = value
        got = c.attend(q, out=torch.zeros_like(before))
        hit = torch.zeros((n, heads, dh), dtype=torch.bool, device="cuda")
        hit[at - cached:, :heads // kv, 7] = True
        assert torch.equal(got.isnan(), hit.view(n, -1))
        assert torch.equal(got[~hit.view(n, -1)], before[~hit.view(n, -1)])
        for i in range(n):
            one = alone(c, 0, i, q, out_type=out_type)
            same = torch.equal(one.nan_to_num(7.0), got[i].nan_to_num(7.0)) and torch.equal(one.isnan(), got[i].isnan())
            assert same, f"row {i}"
        c.v.copy_(keep)


@pytest.mark.parametrize("dtype,heads,kv,dh", HEADS)
@pytest.mark.parametrize("out_type", [None, torch.float32])
def test_rows_beside_a_long_chunk(dtype, heads, kv, dh, out_type):
    """Short chunks in a call with tiles, with outputs in either type: the bits of a single token."""
    print(f"case {dtype} {heads}/{kv}x{dh} {out_type}", flush=True)
    c = Call([(5, 700), (300, 50), (1, 2200), (6, 29)], heads, kv, dh, dtype, seed=9)
    q = climbing(c, 2.0)
    got = c.attend(q, out=torch.zeros_like(q, dtype=out_type or q.dtype))
    B.sdsat_paged_status(c.handle)
    for b in (0, 2, 3):
        for i in range(c.seqs[b][0]):
            same = torch.equal(got[c.start[b] + i], alone(c, b, i, q, out_type=out_type))
            assert same, f"row {i} of sequence {b}"
