"""Tensors that calls on a paged cache and logit rules refuse before they reach the library: types, shapes, rows, strides.
Without a device: a call whose tensors fit gets as far as the library's own word about the handle, which is NULL here."""
import ctypes

import pytest

from paper_2403_18647_amd import binding as B

torch = pytest.importorskip("torch")

HEADS, KV, DH, PAGES, ROWS = 4, 2, 64, 5, 8
POOL = {B.DTYPE_BF16: torch.bfloat16, B.DTYPE_FP32: torch.float32}


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


class Handle(ctypes.c_void_p):
    pass


def handle(code):
    h = Handle()
    h.limits = B._PagedLimits(B.sdsat_paged_config(HEADS, KV, DH, code, PAGES, ROWS, 3, 160), torch.zeros(1))
    return h


def batch(rows=ROWS):
    return B.paged_batch(i32(3), i32(2), i32(2, 5), rows, 4, 100)


def append(code, **kw):
    t = POOL[code]
    a = dict(k=torch.zeros(PAGES, KV, 32, DH, dtype=t), v=torch.zeros(PAGES, KV, DH, 32, dtype=t),
             x=torch.zeros(ROWS, (HEADS + 2 * KV) * DH, dtype=torch.bfloat16), pos=i32(ROWS), q_gain=torch.zeros(DH),
             k_gain=torch.zeros(DH), q_out=torch.zeros(ROWS, HEADS * DH, dtype=t))
    rows = kw.pop("rows", ROWS)
    a.update(kw)
    B.sdsat_paged_append(handle(code), batch(rows), **a)


def attend(code, **kw):
    t = POOL[code]
    a = dict(k=torch.zeros(PAGES, KV, 32, DH, dtype=t), v=torch.zeros(PAGES, KV, DH, 32, dtype=t),
             q=torch.zeros(ROWS, HEADS * DH, dtype=t), mask=torch.zeros(ROWS, dtype=torch.int64),
             out=torch.zeros(ROWS, HEADS * DH, dtype=t))
    rows = kw.pop("rows", ROWS)
    a.update(kw)
    B.sdsat_paged_attention(handle(code), batch(rows), **a)


def other(code):
    return POOL[1 - code]


@pytest.mark.parametrize("code", [B.DTYPE_BF16, B.DTYPE_FP32])
def test_tensors_that_do_not_fit_a_call(code):
    t, o = POOL[code], other(code)
    kv = [("pages", dict(k=torch.zeros(PAGES - 1, KV, 32, DH, dtype=t))), ("pages", dict(v=torch.zeros(PAGES - 1, KV, DH, 32, dtype=t))),
          ("type", dict(k=torch.zeros(PAGES, KV, 32, DH, dtype=o))), ("type", dict(v=torch.zeros(PAGES, KV, DH, 32, dtype=o))),
          ("K's layout for V", dict(v=torch.zeros(PAGES, KV, 32, DH, dtype=t))), ("heads", dict(k=torch.zeros(PAGES, 1, 32, DH, dtype=t))),
          ("flat", dict(k=torch.zeros(PAGES * KV * 32 * DH, dtype=t))),
          ("order", dict(k=torch.zeros(PAGES, 32, KV, DH, dtype=t).transpose(1, 2)))]
    rows = lambda n, w, d: torch.zeros(n, w, dtype=d)
    for what, kw in kv + [
            ("no output", dict(q_out=None)), ("output's type", dict(q_out=rows(ROWS, HEADS * DH, o))),
            ("output's rows", dict(q_out=rows(ROWS - 1, HEADS * DH, t))), ("output's columns", dict(q_out=rows(ROWS, HEADS * DH - 8, t))),
            ("x's type", dict(x=rows(ROWS, 512, torch.float16))), ("x's rows", dict(x=rows(ROWS - 1, 512, t))),
            ("x's columns", dict(x=rows(ROWS, 504, t))), ("x's order", dict(x=rows(512, ROWS, t).t())), ("x's shape", dict(x=rows(1, ROWS * 512, t)[0])),
            ("positions of 64 bits", dict(pos=torch.zeros(ROWS, dtype=torch.int64))), ("positions", dict(pos=i32(ROWS - 1))),
            ("positions' stride", dict(pos=i32(2 * ROWS)[::2])), ("gain's type", dict(q_gain=torch.zeros(DH, dtype=torch.bfloat16))),
            ("gain's length", dict(k_gain=torch.zeros(DH - 1)))]:
        with pytest.raises(ValueError):
            append(code, **kw)
            pytest.fail(what)
    for what, kw in kv + [
            ("queries' type", dict(q=rows(ROWS, HEADS * DH, o))), ("queries' rows", dict(q=rows(ROWS - 1, HEADS * DH, t))),
            ("queries' columns", dict(q=rows(ROWS, HEADS * DH - 1, t))), ("no output", dict(out=None)),
            ("output's type", dict(out=rows(ROWS, HEADS * DH, torch.float16))), ("output's rows", dict(out=rows(2, HEADS * DH, t))),
            ("output's order", dict(out=rows(HEADS * DH, ROWS, t).t())), ("masks of 32 bits", dict(mask=i32(ROWS))),
            ("masks", dict(mask=torch.zeros(ROWS - 1, dtype=torch.int64)))]:
        with pytest.raises(ValueError):
            attend(code, **kw)
            pytest.fail(what)


@pytest.mark.parametrize("code", [B.DTYPE_BF16, B.DTYPE_FP32])
def test_tensors_that_fit_reach_the_library(code):
    t = POOL[code]
    wide = lambda w, d, n=ROWS: torch.zeros(n, w + 40, dtype=d)[:, 16:16 + w]
    pool = lambda: dict(k=torch.zeros(2, PAGES + 3, KV, 32, DH, dtype=t)[1], v=torch.zeros(PAGES + 3, KV, DH, 32, dtype=t))
    for kw in (dict(), pool(), dict(x=wide(512, torch.float32)), dict(q_out=wide(256, t, ROWS + 3)), dict(pos=None, q_gain=None, k_gain=None),
               dict(k=4096, v=None, pos=4096, q_gain=4096), dict(rows=ROWS + 1), dict(rows=-1), dict(rows=3, x=torch.zeros(3, 512))):
        with pytest.raises(B.SdsatError) as e:
            append(code, **kw)
        assert e.value.code == -1 and "paged is NULL" in str(e.value), kw
    for kw in (dict(), pool(), dict(q=wide(256, t)), dict(out=wide(256, t, ROWS + 3)), dict(mask=None), dict(mask=4096),
               dict(out=torch.zeros(ROWS, 256)), dict(rows=ROWS + 1), dict(rows=-1)):
        with pytest.raises(B.SdsatError) as e:
            attend(code, **kw)
        assert e.value.code == -1 and "paged is NULL" in str(e.value), kw


def test_a_description_by_hand_reaches_the_library():
    d = B.sdsat_paged_batch(256, 256, 256, 2, 5, ROWS, 4, 100)
    q = torch.zeros(ROWS, HEADS * DH)
    with pytest.raises(B.SdsatError):
        B.sdsat_paged_attention(handle(B.DTYPE_FP32), d, 256, 256, q, None, 0, 0.0, q)


@pytest.mark.parametrize("name", ["start", "length", "pages"])
def test_descriptions_of_64_bits(name):
    a = dict(start=i32(3), length=i32(2), pages=i32(2, 5))
    a[name] = a[name].long()
    with pytest.raises(ValueError):
        B.paged_batch(**a, rows=4, max_q=2, max_len=100)


def test_views_of_a_table():
    """Past the columns of a view its last row may end the table."""
    table = i32(2, 9)
    assert B.paged_batch(i32(3), i32(2), table[:, 5:8], 4, 2, 96).pages_ld == 9
    for view in (table[:, 5:8], table[1:, 5:8]):
        with pytest.raises(ValueError):
            B.paged_batch(i32(1 + view.shape[0]), i32(view.shape[0]), view, 4, 2, 97)
    B.paged_batch(i32(3), i32(2), table, 4, 2, 10 ** 6)   # refused by the calls


@pytest.mark.parametrize("name,value", [("history", torch.int64), ("history_len", torch.int64), ("prompt_len", torch.int64),
                                        ("tokens", torch.int64), ("allowed", torch.int64), ("mask", torch.int32),
                                        ("penalties", torch.float64), ("bias", torch.bfloat16)])
def test_rules_of_other_types(name, value):
    shapes = dict(history=(2, 9), history_len=(2,), prompt_len=(2,), tokens=(2, 3), allowed=(6, 4), mask=(6,), penalties=(3, 2), bias=(2, 100))
    with pytest.raises(ValueError):
        B.logit_rules(**{name: torch.zeros(shapes[name], dtype=value)})


def test_logits_of_other_types():
    z = torch.zeros(2, 64)
    rules = B.logit_rules()
    for logits, out in ((z.bfloat16(), z), (z, z.double()), (z.t(), z)):
        with pytest.raises(ValueError):
            B.sdsat_adjust_logits(None, 1, 2, logits, rules, out)
    with pytest.raises(B.SdsatError):
        B.sdsat_adjust_logits(None, 1, 2, z, rules, z)
