"""The loads from global memory to LDS that are written in assembly hold by themselves: the
wait states between a scalar address that a vector instruction writes and the load that
reads it, and m0 named as written.  Read from the compiler's assembly of small kernels that
put the least between the two (no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2609_36222_amd import build as B

KERNELS = r"""
#include "attn.hpp"
#include "ffn.hpp"
using namespace basek;
__global__ void near(const uint32_t *at, int l, uint32_t *out) {
  __shared__ __attribute__((aligned(256))) uint32_t lds[1024];
  const char *base = lane_at(at[threadIdx.x], at[64 + threadIdx.x], l);
  glb_to_lds(base, threadIdx.x * 16, lds_addr(lds));
  wait_vm<0>();
  out[threadIdx.x] = lds[threadIdx.x];
}
// m0 holds the same before and behind
__global__ void between(const char *p, const char *q, uint32_t *out) {
  __shared__ __attribute__((aligned(256))) uint32_t lds[1024];
  load_lds(make_rsrc(p, 1 << 20), lds, threadIdx.x * 16, 0);
  glb_to_lds(q + threadIdx.x * 16, lds_addr(lds + 512));
  load_lds(make_rsrc(p, 1 << 20), lds, threadIdx.x * 16, 4096);
  wait_vm<0>();
  out[threadIdx.x] = lds[threadIdx.x] + lds[512 + threadIdx.x];
}
"""


@pytest.fixture(scope="module")
def functions(tmp_path_factory):
    try:
        hipcc = B._hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("asm")
    (at / "k.hip").write_text(KERNELS)
    cmd = [hipcc, *B.FLAGS, "--cuda-device-only", "-S", "-I", B.CSRC, str(at / "k.hip"), "-o", str(at / "k.s")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found, name = {}, None
    for line in (at / "k.s").read_text().splitlines():
        line = line.split(";")[0].strip()
        m = re.match(r"_Z\d+(near|between)", line)
        if m and line.endswith(":"):
            name = m[1]
        elif line.startswith("s_endpgm"):
            name = None
        elif name and line and not line.startswith(".") and not line.endswith(":"):
            found.setdefault(name, []).append(line)
    return found


def scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    return {int(operand[1:])} if re.match(r"s\d+$", operand) else set()


def test_wait_states_before_a_scalar_address_is_read(functions):
    lines = functions["near"]
    loads = [i for i, s in enumerate(lines) if re.match(r"global_load_lds_dwordx4 v\d+, s\[", s)]
    assert len(loads) == 1
    need = scalars(lines[loads[0]].split(",")[1].strip())
    states = 0
    for s in reversed(lines[:loads[0]]):
        if s.startswith("v_readlane") and scalars(s.split()[1].rstrip(",")) & need:
            break
        m = re.match(r"s_nop (\d+)", s)
        states += int(m[1]) + 1 if m else 1
    else:
        pytest.fail("no lane's read in front of the load")
    assert states >= 5


def test_m0_is_named(functions):
    """Each of the three loads has m0 set in front of it, the last one again to what it was."""
    sets = 0
    for s in functions["between"]:
        if re.match(r"s_\w+ m0,", s):
            sets += 1
    assert sets == 3
