"""The tiles of sliding-window attention with many rows (csrc/sliding_plan.h), compiled for the CPU: every key that a row sees is in a tile, once; tiles without masks are seen whole by
every row; nothing is read outside the keys; the same for a row tile's keys dealt to several workgroups.  No GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "sliding_plan.h"
#include <cstdio>
#include <cstring>
using namespace slim;
static int fail(const SlidingRows& a, int r0, const char* what) {
    printf("n_q %d n_k %d G %d window %d sinks %d row %d: %s\n", a.n_q, a.n_k, a.G, a.window, a.sinks, r0, what);
    return 1;
}
static int times[4096];
static int check(const SlidingRows& a, int parts) {
    const int rows = a.n_q * a.G, off = a.n_k - a.n_q;
    for (int r0 = 0; r0 < rows; r0 += 256) {
        const SlidingSpan s(a, r0, 256);
        const SlidingTiles whole(s, a.window);
        const int last_row = r0 + 255 < rows ? r0 + 255 : rows - 1, p0 = off + r0 / a.G, p1 = off + last_row / a.G;
        if (s.p0 != p0 || s.p1 != p1) return fail(a, r0, "positions");
        memset(times, 0, a.n_k * sizeof(int));
        for (int split = 0; split < parts; ++split) {
            const int from = (int)((long long)split * whole.all / parts), to = (int)((long long)(split + 1) * whole.all / parts);
            if (from == to) continue;
            const SlidingTiles t = whole.part(from, to);
            if (t.all != to - from || t.left < 1 || t.left > 128 || t.units < 0 || t.apart != (t.units + 3) / 4 ||
                (t.units > 3 && t.units % 4) || (t.units && t.k00 + t.units * 32 > t.start) || t.clean < t.apart || t.clean > t.all || t.masked < t.clean ||
                t.masked > (t.clean == t.all ? t.all : t.all - 1))
                return fail(a, r0, "counts");
            for (int i = 0; i < t.all; ++i) {
                const int n = i == t.all - 1 ? t.left : 128;
                for (int u = 0; u < 4; ++u) {
                    const int idx = 4 * i + u, k0 = idx < t.units ? t.k00 + idx * 32 : t.start + (idx - t.units) * 32, here = n - 32 * u < 32 ? n - 32 * u : 32;
                    if (idx == 0 && k0 != t.k00) return fail(a, r0, "first key");
                    if (idx >= t.units && k0 != t.origin() + 32 * idx) return fail(a, r0, "origin");
                    if (here < 1) break;
                    if (k0 < 0 || k0 + here > a.n_k) return fail(a, r0, "outside");
                    for (int j = k0; j < k0 + here; ++j) ++times[j];
                    // units whose logits the loop without masks forms
                    if (t.masked == t.clean || idx < 4 * t.clean + 1 || idx > 4 * t.masked) continue;
                    if (here < 32) return fail(a, r0, "a short unit without a mask");
                    for (int j = k0; j < k0 + 32; ++j)
                        for (int p = p0; p <= p1; p += p1 > p0 ? p1 - p0 : 1)
                            if (!(j <= p && (j > p - a.window || j < a.sinks))) return fail(a, r0, "mask");
                }
            }
        }
        for (int p = p0; p <= p1; ++p)
            for (int j = 0; j <= p; ++j)
                if ((j > p - a.window || j < a.sinks) && times[j] != 1) return fail(a, r0, "coverage");
    }
    return 0;
}
int main() {
    unsigned x = 12345;
    auto rnd = [&](int n) { x = x * 1664525u + 1013904223u; return (int)((x >> 8) % (unsigned)n); };
    int cases = 0;
    for (int c = 0; c < 4000; ++c) {
        SlidingRows a{};
        a.n_k = 1 + rnd(c % 4 ? 700 : 2500);
        a.n_q = c % 3 ? 1 + rnd(a.n_k) : a.n_k;
        const int heads[6] = {1, 2, 3, 4, 7, 20};
        a.G = heads[rnd(6)];
        a.window = 1 + rnd(c % 5 ? a.n_k : 1 + a.n_k / 8);
        const int few[10] = {0, 1, 4, 32, 33, 64, 90, 97, 128, 130};
        a.sinks = c % 7 ? few[rnd(10)] : rnd(a.n_k + 1);
        if (a.sinks > a.n_k) a.sinks = a.n_k;
        const int most[8] = {1, 1, 2, 3, 5, 8, 17, 64};
        if (check(a, most[rnd(8)])) return 1;
        ++cases;
    }
    printf("%d cases\n", cases);
    return 0;
}
"""


def test_tiles(tmp_path):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(SOURCE)
    subprocess.run([gxx, "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_06447_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "4000 cases", r.stdout


def test_routes(tmp_path):
    """Which tiles a call runs in and over how many workgroups a tile's keys are dealt: the calls whose sides were measured."""
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("no host compiler")
    parts = [((16, 8208, 4, 8, 4096, 64), 0), ((32, 8224, 4, 8, 4096, 64), 0), ((64, 2000, 7, 4, 500, 4), 0), ((1, 32768, 4, 8, 32768, 0), 0), ((1, 1, 1, 1, 1, 0), 0),
             ((512, 8704, 4, 8, 4096, 64), 4), ((2048, 10240, 4, 8, 4096, 64), 1), ((1511, 11367, 7, 4, 11367, 0), 3), ((32768, 32768, 4, 8, 4096, 64), 1),
             ((4096, 4096, 4, 8, 512, 0), 1), ((1024, 1024, 4, 8, 300, 4), 1)]
    splits = [((1, 8193, 4, 8, 4096, 64), 33), ((16, 8208, 4, 8, 4096, 64), 7), ((1, 1, 1, 1, 1, 0), 1), ((2048, 2048, 2, 2, 2048, 0), 1),
              ((1, 32768, 4, 8, 100, 4), 1), ((64, 8000, 4, 8, 256, 4), 1), ((1, 32768, 4, 8, 256, 64), 3)]
    src, exe = tmp_path / "routes.cpp", tmp_path / "routes"
    text = '#include "sliding_plan.h"\n#include <cstdio>\nusing namespace slim;\nint main() {\n'
    for args, _ in parts:
        text += f'    printf("%d\\n", sliding_parts({", ".join(map(str, args))}));\n'
    for args, _ in splits:
        text += f'    printf("%d\\n", sliding_splits({", ".join(map(str, args))}, 128));\n'
    src.write_text(text + "}\n")
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2508_06447_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [w for _, w in parts + splits]
