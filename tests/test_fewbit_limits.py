"""Limits of the few-bit calls that the host checks by itself (CPU; nothing is launched)."""
import os
import subprocess

import numpy as np
import pytest

import paper_2402_10876_amd as tw
from paper_2402_10876_amd.build import FLAGS, HIPCC

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

P = 0x10000        # never dereferenced


def _status(f, *a):
    with pytest.raises(tw.TwError) as e:
        f(*a)
    return e.value.status


@pytest.mark.parametrize("M", [(1 << 27) + 1, 1 << 28, (1 << 31) - 16])
def test_scaled_int8_product_of_more_than_the_most_tokens(M):
    """M <= 2^27 holds for every few-bit call; 2^27 itself goes on to the next check (the weight is not uploaded)."""
    w = tw.tw_pack_i8_host(np.ones((1, 70), np.int8), np.ones((1, 70), np.uint8), 64)
    ld = -(-M // 16) * 16
    assert _status(tw.tw_gemm_i8_scaled, P, M, ld, w, P, P, 2 * P, ld) == 3
    assert _status(tw.tw_gemm_i8_scaled, P, 1 << 27, 1 << 27, w, P, P, 2 * P, 1 << 27) == 6
    w.free()


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_a_dimension_of_2_32_threads_is_no_failure_of_the_runtime(tmp_path):
    """launch_kernel says hipErrorInvalidValue (which the calls turn into TW_ERR_UNSUPPORTED) before it asks the runtime.  The
    program sees no device, so that nothing can be launched: what passes the check ends as hipErrorNoDevice."""
    src, exe = tmp_path / "driver.hip", tmp_path / "driver"
    src.write_text(r"""
#include <cstdio>
#include "launch.h"
__global__ void nothing(int) {}
int main() {
  int n = 0;
  if (hipGetDeviceCount(&n) == hipSuccess && n > 0) { std::printf("a device\n"); return 2; }
  const unsigned grids[][3] = {{1u << 24, 256, 1}, {(1u << 24) - 1, 256, 0}, {1u << 22, 1024, 1}, {(1u << 22) - 1, 1024, 0}, {0xffffffffu, 64, 1}, {1, 64, 0}};
  int fails = 0;
  for (auto& g : grids)
    fails += (twg::launch_kernel(nothing, dim3(g[0]), dim3(g[1]), nullptr, 1) == hipErrorInvalidValue) != (g[2] != 0);
  std::printf("fails=%d\n", fails);
  return fails != 0;
}
""")
    r = subprocess.run([HIPCC, *[f for f in FLAGS if f not in ("-shared", "-fPIC")], "-I", os.path.join(ROOT, "paper_2402_10876_amd", "csrc"),
                        str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60, env=env)
    assert r.returncode == 0 and "fails=0" in r.stdout, (r.returncode, r.stdout[-2000:], r.stderr[-2000:])
