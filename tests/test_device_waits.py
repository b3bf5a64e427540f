"""The waits of the attention kernels are waits for the compiler too: no LDS access moves over one.  The wait is a
compiler builtin that counts as an access to any memory, which the kernels rely on where a direct load into LDS, which
the compiler does not see, has changed what it reads next (compiled for the GPU, read as assembly; nothing runs)."""
import re
import subprocess

import pytest

from paper_2609_07883_amd import build

SOURCE = r"""
#include "attn_device.h"
using namespace slw;
extern "C" __global__ void loads(const uint32_t* src, uint32_t* out) {
    __shared__ __attribute__((aligned(16))) uint32_t x[256];
    load_lds16(src + 4 * threadIdx.x, x);
    const uint32_t before = x[threadIdx.x];
    wait_vmcnt<0>();
    out[threadIdx.x] = 3 * before + x[threadIdx.x];
}
extern "C" __global__ void stores(const uint32_t* src, uint32_t* out) {
    __shared__ uint32_t x[256];
    x[threadIdx.x] = src[0];
    wait_lgkmcnt0();
    x[threadIdx.x] = src[1];
    barrier_only();
    out[threadIdx.x] = x[threadIdx.x ^ 1];
}
"""


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    d = tmp_path_factory.mktemp("waits")
    (d / "waits.hip").write_text(SOURCE)
    r = subprocess.run([build.HIPCC, *build.HIP_FLAGS, "--offload-device-only", "-S", str(d / "waits.hip"), "-o",
                        str(d / "waits.s")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    text = (d / "waits.s").read_text()
    return {k: re.search(rf"^{k}:(.*?)s_endpgm", text, re.S | re.M).group(1) for k in ("loads", "stores")}


def _ops(text, pattern):
    return [m.group(0) for m in re.finditer(pattern, text)]


def test_lds_read_after_a_wait_for_loads(assembly):
    """A value read before the wait is not taken for the one after it, which a direct load has changed."""
    assert _ops(assembly["loads"], r"global_load_lds_dwordx4|ds_read|vmcnt\(0\)")[:4] == [
        "global_load_lds_dwordx4", "ds_read", "vmcnt(0)", "ds_read"]


def test_lds_write_before_a_wait_for_lds(assembly):
    """A write before the wait is made before it, though another one follows."""
    assert len(_ops(assembly["stores"], r"ds_write")) == 2
