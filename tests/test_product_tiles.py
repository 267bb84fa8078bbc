"""The tiles that products of 8-bit integers are done in (csrc/wz_int8_tile.h), asked for on the host: a small program
compiled against the header, whose launches print the tile instead.  No GPU needed."""
import re
import subprocess

import pytest

import tile_cases as tc
from paper_2607_23265_amd.csrc import build

PROBE = r"""
#include <cstdio>
#include <hip/hip_runtime.h>
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(...) std::printf("%s;", __PRETTY_FUNCTION__)
#define hipGetLastError() hipSuccess
#include "wz_int8_tile.h"
template <int EPI>
hipError_t ask(const wz::MatmulArgs& p, int bf16) {
  return bf16 ? wz::matmul<uint16_t, EPI>(p, nullptr) : wz::matmul<float, EPI>(p, nullptr);
}
int main() {
  int epi, bf16, act, M, N, K, bad = 0;
  while (scanf("%d %d %d %d %d %d", &epi, &bf16, &act, &M, &N, &K) == 6) {
    wz::MatmulArgs p{};
    p.M = M, p.N = N, p.K = K, p.activation = act;
    bad |= (epi == 1 ? ask<wz::kRich>(p, bf16) : ask<wz::kGated>(p, bf16)) != hipSuccess;
    std::printf("\n");
  }
  return bad;
}
"""
ACT = {None: 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}
TILE = re.compile(r"BM = (\d+), BN = (\d+), WM = \d+, WN = \d+, ST = (\d+), KS = (\d+), EPI = \d, KB = (\d+)")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    src, exe = str(d / "tiles.hip"), str(d / "tiles")
    with open(src, "w") as f:
        f.write(PROBE)
    subprocess.run([build.hipcc(), "-O1", "-std=c++17", "--offload-host-only", "-I", build.INCLUDE, "-I", build.HERE, src,
                    "-o", exe], check=True, capture_output=True, timeout=300)

    def run(epilogue, cases):
        """Tiles of each (bf16, activation, M, N, K)."""
        text = "".join(f"{epilogue} {int(b)} {ACT[a]} {M} {N} {K}\n" for b, a, M, N, K in cases)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60)
        return [["%sx%s/%s/%s/%s" % TILE.search(x).groups() for x in line.split(";") if x] for line in r.stdout.splitlines()]

    return run


@pytest.mark.parametrize("epilogue,cases", [(1, tc.RICH), (2, tc.GATED)])
def test_cases_reach_their_tiles(plan, epilogue, cases):
    for bf16 in (True, False):
        got = plan(epilogue, [(bf16, *c[:4]) for c in cases])
        assert got == [c[4] for c in cases]


@pytest.mark.parametrize("epilogue,cases", [(1, tc.RICH), (2, tc.GATED)])
def test_every_tile_is_reached(plan, epilogue, cases):
    """By a case of its own, and no product of ordinary size by another tile."""
    assert {c[4][0] for c in cases if len(c[4]) == 1} == set(tc.TILES)
    sizes = [(True, act, M, N, K) for act in (None, "silu", "gelu") for M in (1, 33, 64, 300, 1286, 2400, 9459, 12544)
             for N in (100, 1152, 3584, 14336) for K in (144, 1152, 3584, 14336)]
    used = [t for tiles in plan(epilogue, sizes) for t in tiles]
    assert set(used) <= set(tc.TILES) and len(used) >= len(sizes)
