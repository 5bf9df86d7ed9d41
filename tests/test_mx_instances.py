"""Which kernel instances the 4-bit layers of test_gpu_mx.py take, by the rules of the
library's own header compiled here: a line that moves must not leave one untested."""
import ctypes
import os
import subprocess

import pytest

from paper_2609_36222_amd import build

N_CU = 256
SOURCE = """
#include "internal.hpp"
using namespace basek;
extern "C" int gateup(int B, int I, int K, int budget, int ns) {
  return mx_gateup_shape(B, I, K, budget, ns, %d);
}
extern "C" int few(int B, int K, int budget, int ns, int d, int I) { return mx_few(B, K, budget, ns, d, I); }
extern "C" int loads(int B) { return mx_row_loads(B); }
extern "C" int shares(int B, int K, int budget, int ns, int d, int I) {
  return mx_down_shares(B, K, budget, ns, d, I);
}
extern "C" int parts(int B) { return mx_parts(B); }
extern "C" int counts(int n_kept, int nx) { return mx_pick_counts(n_kept, nx); }
extern "C" int few_plan_b() { return FEW_PLAN_B; }
extern "C" int two_b() { return MX_TWO_B; }
""" % N_CU


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    pytest.importorskip("torch")     # its HIP runtime, which the header's library needs
    where = tmp_path_factory.mktemp("rules")
    src, out = where / "rules.cpp", where / "rules.so"
    src.write_text(SOURCE)
    subprocess.check_call([build._hipcc(), "-w", "-std=c++17", "-shared", "-fPIC", "--cuda-host-only",
                           "-I", os.path.abspath(build.CSRC), "-x", "hip", str(src), "-o", str(out)])
    return ctypes.CDLL(str(out))


def shapes():
    pytest.importorskip("torch")
    import test_gpu_mx as g
    return g.SHAPES + g.INSTANCES


def test_every_product_instance_has_a_case(rules):
    gateup, down = set(), set()
    for d, E, K, I, B, budget, flags, ns, _, _, _ in shapes():
        bc = min(budget, E)
        gateup.add(rules.gateup(B, I, K, bc, ns))
        if rules.few(B, K, bc, ns, d, I):
            down.add(("with the combine", rules.loads(B)))
        else:
            tiles = 1 if B <= 16 else 2 if B <= rules.two_b() else 4
            down.add((tiles, rules.shares(B, K, bc, ns, d, I) > 1))
    assert gateup == set(range(5))
    assert down == {("with the combine", n) for n in (1, 2, 4)} | {(n, s) for n in (1, 2, 4) for s in (False, True)}


def test_every_plan_instance_has_a_case(rules):
    """k_plan_few (fused, few tokens) and k_plan_given (staged, no dropped routes), by
    experts a lane, tokens a wavefront and the way kept experts are ranked."""
    few, given, dropped = set(), set(), 0
    for d, E, K, I, B, budget, flags, ns, _, _, _ in shapes():
        kept = min(budget, E, B * K)
        lane, count = 1 if E <= 64 else 2 if E <= 128 else 4, bool(rules.counts(kept, min(K, kept)))
        if not count and K >= 8:
            # a union that is as large or, with fewer experts, still beyond the line
            assert B * K >= 100 and not rules.counts(3 * kept // 4, K)
        if B <= rules.few_plan_b() and not flags & 2:
            few.add((lane, count))
        if not rules.parts(B) and not flags & 2:
            given.add((lane, B <= 16, count))
        dropped += bool(flags & 2)
    assert few == {(n, m) for n in (1, 2, 4) for m in (False, True)}
    assert given == {(n, s, m) for n in (1, 2, 4) for s in (False, True) for m in (False, True)}
    assert dropped
