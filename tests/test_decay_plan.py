"""The plan of linear attention's prompts (csrc/wz_decay_prompt.hip), asked for on the host by a small program compiled
against its header, and what the bounds on its states would catch.  No GPU needed."""
import os
import subprocess

import numpy as np
import pytest

import decay_cases as dc
import libutil
from paper_2607_23265_amd import wavezip as wz
from paper_2607_23265_amd.csrc import build
from serve_util import bf16

PROBE = r"""
#include <cstdio>
#include "wz_serve.h"
int main() {
  int batch, tokens, most, heads, dim;
  while (scanf("%d %d %d %d %d", &batch, &tokens, &most, &heads, &dim) == 5) {
    wz_states z{};
    wz_ragged r{};
    z.slots = 1, z.heads = heads, z.head_dim = dim;
    r.batch = batch, r.tokens = tokens, r.max_tokens = most;
    const wz::DecayPlan p = wz::decay_plan(z, r);
    std::printf("%d %d %d\n", p.token, p.runs, p.join);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    libutil.ensure_built()
    d = tmp_path_factory.mktemp("plan")
    src, exe = str(d / "plan.hip"), str(d / "plan")
    with open(src, "w") as f:
        f.write(PROBE)
    libdir = os.path.dirname(wz.LIB_PATH)
    subprocess.run([build.hipcc(), "-O1", "-std=c++17", "--offload-host-only", "-I", build.INCLUDE, "-I", build.HERE,
                    src, f"-L{libdir}", f"-l:{os.path.basename(wz.LIB_PATH)}", f"-Wl,-rpath,{libdir}", "-o", exe],
                   check=True, capture_output=True, timeout=300)

    def run(new, heads, dim, behind=3, most=None):
        r = subprocess.run([exe], input=f"{len(new)} {sum(new) + behind} {most or max(new)} {heads} {dim}\n",
                           capture_output=True, text=True, check=True, timeout=60)
        return list(map(int, r.stdout.split()))

    return run


def chunks(new):
    return [-(-n // 64) for n in new]


@pytest.mark.parametrize("new,held,heads,kv,dim,behind", dc.JOINED)
def test_joined_cases_are_joined(plan, new, held, heads, kv, dim, behind):
    token, runs, join = plan(new, heads, dim, behind)
    assert not token and join
    per = sum(chunks(new)) / min(runs, sum(chunks(new)))
    assert per >= 1.9 and max(chunks(new)) / per > 16  # runs of the longest sequence


def test_others_are_joined(plan):
    for new, _, heads, _, dim, behind in dc.PADDED:
        _, runs, join = plan(new, heads, dim, behind, sum(new) + behind)
        assert join and runs > sum(chunks(new)) // 2
    for new, dim in dc.AGREE:
        assert plan(new, 3, dim)[2]
    assert plan([9459], 28, 128, 0)[2]  # (one long video's prompt)


@pytest.mark.parametrize("n,rate", [(200, -8), (1286, -8), (1286, -3), (9000, -8), (9000, -5)])
def test_values_in_two_parts_would_be_noticed(n, rate):
    """A state whose sums took the decayed values in two parts of bf16 and not three is off by more than the bound that
    the states are held to (state_norm_bound); in three parts, with sums in fp32 by 16 tokens, it is within."""
    from test_gpu_serve_decay_joined import state_norm_bound
    r = np.random.default_rng(n)
    k, v = bf16(r.normal(size=(n, 64))).astype(np.float64), bf16(r.normal(size=(n, 64)))
    w = np.exp(-np.exp(rate) * np.arange(n - 1, -1, -1)).astype(np.float32)
    x = v * w[:, None]

    def cut(x):  # to bf16, towards zero
        return (np.ascontiguousarray(x).view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)

    parts = [cut(x), cut(x - cut(x))]
    parts.append(x - parts[0] - parts[1])
    assert (cut(parts[2]) == parts[2]).all() and (sum(p.astype(np.float64) for p in parts) == x).all()
    want = k.T @ x.astype(np.float64)
    off = k.T @ (parts[0].astype(np.float64) + parts[1]) - want
    bound = state_norm_bound([n], 0)
    assert np.linalg.norm(off) > 1.5 * bound * np.linalg.norm(want)
    S = np.zeros((64, 64), np.float32)
    for t in range(0, n, 16):
        for p in parts:
            S = (S.astype(np.float64) + k[t:t + 16].T @ p[t:t + 16].astype(np.float64)).astype(np.float32)
    assert np.linalg.norm(S - want) < bound * np.linalg.norm(want)
