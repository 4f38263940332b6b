"""Cache reordering, shared-prefix attention and token log probabilities: what the host refuses, and the launch
plans (tests/operator_check.cpp).  No device."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2403_18647_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.join(os.path.dirname(HERE), "paper_2403_18647_amd")
LIB = os.path.join(PKG, "libsdsat.so")
ROCM = "/opt/rocm"


@pytest.mark.parametrize("name,args", [
    ("sdsat_kv_reorder", (None, 1, None, 0)),
    ("sdsat_cache_ptr", (None, 0, None, None)),
    ("sdsat_attention_shared", (None, 0, 2, 1, 2, None, None, None, None)),
    ("sdsat_forward_block_shared", (None, 2, 1, 2, None, None, None, None)),
    ("sdsat_token_logprobs", (None, 1, 1, None, None, 1.0, 0, None, None, None, None)),
])
def test_null_context(name, args):
    assert getattr(B.lib(), name)(*args) == -1
    assert b"ctx" in B.lib().sdsat_last_error(None)


@pytest.mark.parametrize("batch,group,lens", [(4, 2, [1]), (4, 2, [1, 2, 3]), (4, 0, [1])])
def test_one_prefix_length_per_group(batch, group, lens):
    with pytest.raises(ValueError):
        B._prefix_lens(batch, group, lens)


def test_prefix_lengths_become_a_c_array():
    a = B._prefix_lens(6, 3, [5, 70])
    assert isinstance(a, ctypes.Array) and list(a) == [5, 70]


@pytest.mark.skipif(not os.path.exists(LIB) or shutil.which("g++") is None, reason="library or g++ missing")
def test_plans_and_launch_refusals(tmp_path):
    exe = str(tmp_path / "operator_check")
    cmd = ["g++", "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include",
           f"-I{os.path.join(PKG, 'csrc')}", os.path.join(HERE, "operator_check.cpp"), LIB,
           f"-Wl,-rpath,{PKG}", f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok (0 failed)"), r.stdout[-3000:] + r.stderr[-2000:]
