"""Host code of the operators around the layer, compiled by itself and run without a GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_01956_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def run_host(tmp_path, source):
    """Compiles a host program against the operators' headers; its output's lines."""
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(source)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__",
                    "-I", os.path.join(ROCM, "include"), "-I", CSRC, str(src), "-o", str(exe)],
                   check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True,
                          text=True).stdout.splitlines()


PIECES = r"""
#include "kan_ops.h"
#include <cstdio>
int main() {
    struct { long long rows; unsigned tiles; long long stride, dstride; int entropy; } cases[] = {%s};
    for (auto& c : cases) {
        kan::LogprobGradArgs a = {};
        a.z = (const void*)0; a.dz = (void*)0;
        a.rows = c.rows; a.tiles = c.tiles; a.stride = c.stride; a.dstride = c.dstride;
        if (c.entropy) a.entropy = a.dentropy = (const float*)4096;
        kan::logprob_grad_pieces(a, 2, [&](const kan::LogprobGradArgs& p, int grid) {
            printf("%%lld %%u %%d %%lld %%lld %%lld %%lld %%lld %%lld\n", (long long)p.rows, p.items, grid,
                   (long long)p.z, (long long)p.dz, (long long)p.targets, (long long)p.stats,
                   (long long)p.dlogp, (long long)p.entropy);
            return hipSuccess;
        });
        printf("end %%d\n", kan::logprob_groups(c.rows * c.tiles));
    }
}
"""


def test_rows_past_one_launch(tmp_path):
    """A launch holds fewer than 2^32 work-items of 256 per workgroup, four tiles a workgroup:
    rows around that limit go in pieces that follow one another in every argument, and the
    forward's workgroups stay within it."""
    most = 4 * ((1 << 24) - 1)
    cases = [(1, 1, 300, 300, 1), (most - 1, 1, 257, 260, 1), (most, 1, 257, 257, 0),
             (most + 1, 1, 257, 300, 1), (1 << 26, 1, 257, 257, 1), (3 * most + 5, 1, 512, 513, 0),
             (most // 3 + 1, 3, 5000, 6001, 1), (1000, 1 << 19, 1 << 30, 1 << 30, 0)]
    text = ", ".join("{%d, %d, %d, %d, %d}" % c for c in cases)
    lines = iter(run_host(tmp_path, PIECES % text))
    for rows, tiles, stride, dstride, entropy in cases:
        done = launches = 0
        for line in lines:
            if line.startswith("end"):
                assert int(line.split()[1]) == min((rows * tiles + 3) // 4, (1 << 24) - 1)
                break
            n, items, grid, z, dz, targets, stats, dlogp, ent = map(int, line.split())
            assert n > 0 and items == n * tiles and 4 * (grid - 1) < items <= 4 * grid
            assert grid * 256 < 1 << 32
            assert (z, dz) == (2 * done * stride, 2 * done * dstride)
            assert (targets, stats, dlogp) == (8 * done, 8 * done, 4 * done)
            assert ent == (4096 + 4 * done if entropy else 0)
            done += n
            launches += 1
        assert done == rows and launches == -(-rows // (most // tiles))
