"""Limits of cache reordering, shared-prefix attention and token log probabilities that need no device
(tests/operator_limits_check.cpp), and the memory that they take."""
import os
import shutil
import subprocess

import pytest

from paper_2403_18647_amd import binding as B
from paper_2403_18647_amd import synth

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.join(os.path.dirname(HERE), "paper_2403_18647_amd")
LIB = os.path.join(PKG, "libsdsat.so")
ROCM = "/opt/rocm"


@pytest.mark.skipif(not os.path.exists(LIB) or shutil.which("g++") is None, reason="library or g++ missing")
def test_limits(tmp_path):
    exe = str(tmp_path / "operator_limits_check")
    cmd = ["g++", "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include",
           f"-I{os.path.join(PKG, 'csrc')}", os.path.join(HERE, "operator_limits_check.cpp"), LIB,
           f"-Wl,-rpath,{PKG}", f"-L{ROCM}/lib", "-lamdhip64", f"-Wl,-rpath,{ROCM}/lib", "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok (0 failed)"), r.stdout[-3000:] + r.stderr[-2000:]


@pytest.mark.parametrize("shape,batch,block,ctx,without", [
    (synth.TINY, 64, 64, 128, 107137792), (synth.TINY, 4, 6, 128, 9938176), (synth.LLAMA7B, 8, 64, 1312, 18871766016),
    (synth.LLAMA7B, 64, 64, 1312, 58342329344), (synth.LLAMA7B, 16, 1024, 4096, 51933424640),
    (synth.LLAMA13B, 16, 64, 2048, 52874548224)])
def test_contexts_are_no_larger_for_shared_attention(shape, batch, block, ctx, without):
    """Its parts lie over scratch that is idle meanwhile: a context takes at most 1 MB more than `without` it, reordering
    and log probabilities (sizes of the library without the three)."""
    size = B.sdsat_query_sizes(B.make_config(shape, max_batch=batch, max_ctx=ctx, max_block=block))
    assert size <= without + 1_000_000
