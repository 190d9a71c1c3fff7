"""The process-wide sharing switch, on the CPU: a call reads it once, so that the workspace is checked
for the way that is launched, also if another thread sets the switch in the middle of the call.  The
library runs with the launches and the switch replaced by recorders (no GPU is seen or needed)."""
import os
import shutil
import subprocess
import sys

import pytest

SHIM = r"""
#include "cache_attention.cuh"
namespace {
int reads = 0, script[2] = {0, 0}, plain = 0, shared = 0;
}
namespace ssd {
// the switch: script[0] the first time a call reads it, script[1] from then on
int32_t cache_sharing() { return script[reads++ > 0]; }
cudaError_t launch_cache_attention(const CacheAttnArgs&, void*, cudaStream_t) {
  ++plain;
  return cudaErrorNotSupported;
}
cudaError_t launch_cache_attention_tc(const CacheAttnArgs& a, const CacheAttnLaunch&, cudaStream_t, bool) {
  ++(a.groups > 0 ? shared : plain);
  return cudaErrorNotSupported;
}
cudaError_t launch_cache_attention_stack(const CacheAttnArgs&, const CacheAttnLaunch&, int32_t, cudaStream_t) {
  ++shared;
  return cudaErrorNotSupported;
}
}  // namespace ssd
extern "C" void shim_begin(int first, int then) {
  script[0] = first, script[1] = then;
  reads = plain = shared = 0;
}
extern "C" int shim_plain() { return plain; }
extern "C" int shim_shared() { return shared; }
"""

RUN = r"""
import ctypes, sys
import paper_2606_20543_gb300 as lib
so, shim = lib.load(), ctypes.CDLL(sys.argv[1])
F, NEVER, ALWAYS, CUDA, WORKSPACE = 0x1000, 2, 1, 4, 7
g = ctypes.byref(lib.grid(16, 16, 32))

def need(how, B, D, Hq):
    shim.shim_begin(how, how)
    return so.ssd_cache_attention_shared_workspace(B, 2, Hq, 2, 64, D, 4096, 1024)

def call(first, then, B, D, Hq, n):
    c = lib.BlockCache(8, 16, 2, 64, F, F, F, F)
    shim.shim_begin(first, then)
    s = so.ssd_cache_attention_shared(g, ctypes.byref(c), B, 2, F, F, 64, Hq, F, F, None, None, D, F, 256, F,
                                      0.0, F, None, F, n, F, None)
    return s, shim.shim_plain(), shim.shim_shared()

# few rows a group and many, a token and drafts
for B, D, Hq in ((4, 1, 4), (64, 1, 8), (6, 40, 4)):
    never, always = need(NEVER, B, D, Hq), need(ALWAYS, B, D, Hq)
    assert never < always, (never, always)
    # each way in the workspace that was asked for under it
    assert call(NEVER, NEVER, B, D, Hq, never) == (CUDA, 1, 0)
    assert call(ALWAYS, ALWAYS, B, D, Hq, always) == (CUDA, 0, 1)
    assert call(ALWAYS, ALWAYS, B, D, Hq, always - 1) == (WORKSPACE, 0, 0)
    # set in the middle of the call: the way that the workspace was checked for
    assert call(NEVER, ALWAYS, B, D, Hq, never) == (CUDA, 1, 0)
    assert call(ALWAYS, NEVER, B, D, Hq, always) == (CUDA, 0, 1)
    assert call(ALWAYS, NEVER, B, D, Hq, never) == (WORKSPACE, 0, 0)
print("ok")
"""


def test_a_call_reads_the_switch_once(tmp_path):
    from paper_2606_20543_gb300 import build
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    build.build()
    src, shim = tmp_path / "shim.cu", tmp_path / "shim.so"
    src.write_text(SHIM)
    subprocess.run([build.nvcc()] + build.ARCH + ["-std=c++17", "-Xcompiler", "-fPIC", "-shared", "-I" + build.CSRC,
                    "-I" + os.path.join(build.ROOT, "include"), str(src), "-o", str(shim)], check=True)
    env = dict(os.environ, LD_PRELOAD=str(shim), CUDA_VISIBLE_DEVICES="", PYTHONPATH=build.ROOT)
    r = subprocess.run([sys.executable, "-c", RUN, str(shim)], capture_output=True, text=True, env=env)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
