"""Host code of the operators around the layer, compiled by itself and run without a GPU."""
import os
import shutil
import subprocess
import sys

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


CLASH = r"""
#include "kan_clip_lists.h"
#include <cstdio>
#include <random>
#include <vector>
int main() {
    std::mt19937 rng(7);
    auto draw = [&](int n) { return (int)(rng() %% n); };
    int yes = 0, no = 0;
    for (int round = 0; round < 3000; ++round) {
        const int count = round %% 100 == 0 ? 900 + draw(1400) : 1 + draw(40);
        std::vector<const void*> in(count);
        std::vector<void*> out(count);
        std::vector<int64_t> sizes(count);
        std::vector<int32_t> dtypes(count);
        // pieces of one buffer, side by side, in any order
        std::vector<uintptr_t> at(2 * count);
        uintptr_t p = 4096;
        std::vector<int> order(count);
        for (int t = 0; t < count; ++t) {
            order[t] = t;
            sizes[t] = draw(8) == 0 ? 0 : 1 + draw(60);
            dtypes[t] = draw(2);
        }
        if (round %% 3) std::shuffle(order.begin(), order.end(), rng);
        for (int k = 0; k < count; ++k) {
            const int t = order[k];
            const uintptr_t n = sizes[t] * (dtypes[t] ? 2 : 4);
            in[t] = (const void*)p;
            p += n;
            out[t] = draw(3) ? (void*)in[t] : (void*)p;
            if (out[t] != in[t]) p += n;
        }
        // sometimes a clash: an output or an input moved by a few bytes, or onto another
        const int t = draw(count), u = draw(count);
        switch (draw(6)) {
            case 0: out[t] = (char*)out[t] + 4 * (1 + draw(3)); break;
            case 1: out[t] = out[u]; break;
            case 2: out[t] = (void*)in[u]; break;
            case 3: in[t] = in[u]; break;
            default: break;
        }
        const kan::ClipList l = {count, in.data(), out.data(), sizes.data(), dtypes.data()};
        bool want = false;
        for (int a = 0; a < count && !want; ++a)
            for (int b = 0; b < count && !want; ++b) {
                const int64_t na = sizes[a] * (dtypes[a] ? 2 : 4), nb = sizes[b] * (dtypes[b] ? 2 : 4);
                if (na == 0 || nb == 0) continue;
                auto over = [&](const void* x, const void* y) {
                    return (uintptr_t)x < (uintptr_t)y + nb && (uintptr_t)y < (uintptr_t)x + na;
                };
                if (a != b && over(out[a], out[b])) want = true;
                if (over(out[a], in[b]) && !(a == b && in[a] == out[a])) want = true;
            }
        if (kan::clip_outputs_clash(l) != want || kan::clip_outputs_clash<16>(l) != want ||
            kan::clip_outputs_clash<500>(l) != want) {
            printf("wrong: round %%d count %%d want %%d\n", round, count, (int)want);
            return 0;
        }
        (want ? yes : no) += 1;
    }
    printf("%%d %%d\n", yes, no);
}
"""


def test_overlaps_of_tensor_lists(tmp_path):
    """Lists of up to 2300 tensors, in order and shuffled, with and without a clash of each kind
    (outputs with outputs, outputs with other tensors' inputs, a partial one with its own),
    in one block of outputs and in several, against a comparison of all pairs."""
    line, = run_host(tmp_path, CLASH % ())
    yes, no = map(int, line.split())
    assert yes > 500 and no > 500


STACK = r"""
import sys, threading
from paper_2609_01956_amd import binding as kb
kb.load_library()
count, got = int(sys.argv[1]), []
need = kb.kan_grad_norm_workspace_bytes(count)[1]
g = [(1 << 36) + 64 * (i * 1237 % count) for i in range(count)]
o = [a + (1 << 36) for a in g]
o[-1] = o[0] + 4
args = (g, [16] * count, [kb.KAN_F32] * count, 1.0, 1e-6, o, 1 << 40, need, 1 << 41)
threading.stack_size(128 << 10)
t = threading.Thread(target=lambda: got.append(kb.kan_clip_grad_norm(*args)))
t.start()
t.join()
assert got == [kb.KAN_ERR_INVALID_ARG], got
"""


@pytest.mark.parametrize("count", [2, 12, 16384])
def test_a_small_stack_is_enough(count):
    """A call from a thread of 128 KB (refused on the host for an overlap, the last check)."""
    subprocess.run([sys.executable, "-c", STACK, str(count)], check=True, cwd=ROOT)
