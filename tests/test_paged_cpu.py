"""The paged cache and the logit rules without a device: what the host refuses, rotary frequencies, sizes, plans
(tests/paged_check.cpp)."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest

from paper_2403_18647_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.join(os.path.dirname(HERE), "paper_2403_18647_amd")
LIB = os.path.join(PKG, "libsdsat.so")
ROCM = "/opt/rocm"


def config(**kw):
    c = dict(n_heads=8, n_kv_heads=2, head_dim=128, dtype=1, n_pages=10, max_rows=64, max_batch=4, max_ctx=1000)
    c.update(kw)
    return B.sdsat_paged_config(*[c[n] for n, _ in B.sdsat_paged_config._fields_])


@pytest.mark.parametrize("name,args", [
    ("sdsat_adjust_logits", (None, 1, 1, None, None, None)),
    ("sdsat_paged_append", (None, None, None, None, None, 0, 0, None, None, None, None, 0.0, None, 0)),
    ("sdsat_paged_attention", (None, None, None, None, None, 0, None, 0, 0.0, None, 0, 0)),
    ("sdsat_paged_status", (None,)),
    ("sdsat_paged_query_sizes", (None, None)),
    ("sdsat_paged_init", (None, None, 0, None, None)),
    ("sdsat_rope_init", (0, 64, 1e4, 0, 1.0, 0.0, 1.0, 4.0, 1.0, None)),
])
def test_null_arguments(name, args):
    assert getattr(B.lib(), name)(*args) == -1
    assert b"NULL" in B.lib().sdsat_last_error(None)
    assert B.lib().sdsat_paged_last_error(None) == B.lib().sdsat_last_error(None)


def test_destroying_nothing():
    assert B.lib().sdsat_paged_destroy(None) == 0


@pytest.mark.parametrize("field,value,code", [
    ("n_heads", 0, -1), ("n_kv_heads", 0, -1), ("n_kv_heads", 3, -1), ("n_kv_heads", 16, -1), ("head_dim", 96, -5), ("dtype", 2, -1),
    ("n_pages", 0, -1), ("max_rows", 0, -1), ("max_batch", 0, -1), ("max_ctx", 0, -1), ("max_ctx", (1 << 24) + 1, -5),
    ("max_batch", 4097, -5), ("max_rows", (1 << 20) + 1, -5), ("n_heads", 2048, -5), ("wide", (1024, 1024, 1024), -5)])
def test_configs_that_are_refused(field, value, code):
    kw = dict(zip(("n_heads", "n_kv_heads", "max_batch"), value)) if field == "wide" else {field: value}
    with pytest.raises(B.SdsatError) as e:
        B.sdsat_paged_query_sizes(config(**kw))
    assert e.value.code == code
    out = ctypes.c_void_p()
    assert B.lib().sdsat_paged_init(ctypes.byref(config(**kw)), 256, 1 << 40, None, ctypes.byref(out)) == code
    assert out.value is None


def test_workspaces_that_are_refused():
    cfg = config()
    size = B.sdsat_paged_query_sizes(cfg)
    out = ctypes.c_void_p()
    init = B.lib().sdsat_paged_init
    assert init(ctypes.byref(cfg), None, size, None, ctypes.byref(out)) == -1
    assert init(ctypes.byref(cfg), 384 + 128, size - 1, None, ctypes.byref(out)) == -2
    assert init(ctypes.byref(cfg), 128, size, None, ctypes.byref(out)) == -1
    assert out.value is None


def test_sizes():
    """Scratch of one part needs none for parts; long contexts a bounded number of them, pages none at all."""
    one = B.sdsat_paged_query_sizes(config(n_heads=2, max_rows=8, max_ctx=512))
    assert one < 1 << 12
    assert B.sdsat_paged_query_sizes(config(n_pages=10 ** 6)) == B.sdsat_paged_query_sizes(config())
    a, b = (B.sdsat_paged_query_sizes(config(max_rows=8, n_heads=2, max_ctx=c)) for c in (65536, 1 << 24))
    assert a <= b <= 4 * 2 * 64 * 64 * 132 * 4 + 4096


@pytest.mark.parametrize("kw,code", [
    (dict(layout=2), -1), (dict(rot_dims=-8), -5), (dict(rot_dims=12), -5), (dict(rot_dims=136), -5), (dict(base=0.0), -1),
    (dict(base=math.inf), -1), (dict(base=math.nan), -1), (dict(scaling=4), -1), (dict(scaling=1, factor=0.0), -1),
    (dict(scaling=2, factor=-1.0), -1), (dict(scaling=3, ctx=0.0), -1), (dict(scaling=3, low=4.0), -1), (dict(scaling=3, low=math.nan), -1),
    (dict(mscale=math.nan), -1)])
def test_rotary_arguments_that_are_refused(kw, code):
    a = dict(layout=0, rot_dims=64, base=1e4, scaling=0, factor=2.0, ctx=4096.0, low=1.0, high=4.0, mscale=1.0)
    a.update(kw)
    assert B.lib().sdsat_rope_init(*a.values(), ctypes.byref(B.sdsat_rope())) == code


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "parts"])
@pytest.mark.parametrize("rot", [0, 8, 24, 128])
def test_rotary_frequencies(scaling, rot):
    base, factor, ctx, low, high = 5e5, 8.0, 8192.0, 1.0, 4.0
    r = B.sdsat_rope_init("interleaved", rot, base, scaling, factor, ctx, low, high, 1.5)
    assert (r.layout, r.rot_dims, r.mscale) == (1, rot, 1.5)
    for j in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
        f = b ** (-2 * j / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            w = 2 * math.pi / f   # positions of a turn
            if w > ctx / low:
                f /= factor
            elif w > ctx / high:
                s = (ctx / w - low) / (high - low)
                f = (1 - s) * f / factor + s * f
        assert math.isclose(r.turns[j], f / (2 * math.pi), rel_tol=1e-13)
    assert not any(r.turns[rot // 2:])


def test_descriptions_check_their_tensors():
    torch = pytest.importorskip("torch")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    b = B.paged_batch(i32(4), i32(3), i32(3, 7), 20, 5, 200)
    assert (b.batch, b.pages_ld, b.rows, b.max_q, b.max_len) == (3, 7, 20, 5, 200)
    assert B.paged_batch(i32(4), i32(3), i32(3, 9)[:, :7], 20, 5, 200).pages_ld == 9
    for args in [(i32(3), i32(3), i32(3, 7)), (i32(4), i32(3), i32(2, 7)), (i32(4), i32(3), i32(21)), (i32(8)[::2], i32(3), i32(3, 7)),
                 (i32(4), i32(3), i32(7, 3).t())]:
        with pytest.raises(ValueError):
            B.paged_batch(*args, 20, 5, 200)
    bias = torch.zeros(2, 10)
    assert B.logit_rules(bias=bias).bias_ld == 10 and B.logit_rules(bias=bias[:1]).bias_ld == 0 and B.logit_rules(bias=bias[0]).bias_ld == 0
    with pytest.raises(ValueError):
        B.logit_rules(history=i32(6, 2).t())
    with pytest.raises(ValueError):
        B._dtype_code(torch.zeros(2, dtype=torch.float16))
    with pytest.raises(ValueError):
        B._row_stride(torch.zeros(4, 6).t())


@pytest.mark.skipif(not os.path.exists(LIB) or shutil.which("g++") is None, reason="library or g++ missing")
def test_plans_and_launch_refusals(tmp_path):
    exe = str(tmp_path / "paged_check")
    cmd = ["g++", "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include",
           f"-I{os.path.join(PKG, 'csrc')}", os.path.join(HERE, "paged_check.cpp"), LIB,
           f"-Wl,-rpath,{PKG}", f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok (0 failed)"), r.stdout[-3000:] + r.stderr[-2000:]
