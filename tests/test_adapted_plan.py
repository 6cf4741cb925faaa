"""The rules that choose and cut the kernels of the adapted projection, compiled from the header that the library compiles (no GPU)."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(__file__), "..", "paper_2609_34054_b200", "csrc")
SMS, SMEM = 148, 232448
# blocks of a cluster -> clusters that are resident at once, as a B200 reports them
CLUSTERS = "0, 0, 74, 48, 34, 27, 22, 18, 16"
M_ALL = (1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 128, 255, 256, 257, 400, 777, 1024, 2047, 2048, 3001, 4096, 4097, 8192, 16384, 37888, 37889, 100000, 2 ** 24, 2 ** 26)


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("adapted_plan")

    def call(expr, rows):
        src, exe = d / "plan.cpp", d / f"plan_{abs(hash(expr))}"
        if not exe.exists():
            src.write_text('#include <cstdio>\n#include "adapted_plan.h"\nusing namespace precc;\n'
                           f'int main() {{ const int clusters[] = {{{CLUSTERS}}}; long a[5]; '
                           f'while (scanf("%ld %ld %ld %ld %ld", a, a + 1, a + 2, a + 3, a + 4) == 5) {{ {expr} }} (void)clusters; }}\n')
            subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
        text = "\n".join(" ".join(map(str, (list(r) + [0] * 5)[:5])) for r in rows)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout
        return [[int(v) for v in line.split()] for line in out.splitlines()]
    return call


def _shapes():
    return [(M, K, N, r, q) for M in M_ALL for K in (64, 128, 192, 640, 1024, 4096, 14336, 2 ** 20) for N in (8, 24, 136, 1000, 4096, 14336, 2 ** 20)
            for r in (0, 8, 64) for q in (0, 1) if not (q and K % 128)]


def test_every_call_has_a_kernel_that_fits(plan):
    """Every cut covers the call, gives every block of a cluster a k-block, and stays inside shared memory (beside the small shrink kernel where that runs beside it)
    and the grid."""
    for force in (0, 2, 3):
        got = plan(f'AdaptedPlan p = plan_adapted(a[0], a[2], a[1], a[3], a[4], {SMS}, {SMEM}, clusters, {force}); '
                   'printf("%d %d %d %d %d %d %d\\n", p.kernel, p.bn, p.tn, p.ks, p.stages, (int)p.shrink_tc, '
                   'p.kernel == ADAPTED_PAIR ? ap_smem_bytes(p.bn, p.stages) : p.kernel == ADAPTED_TURN ? at_smem_bytes(p.tn, p.ks, p.stages) : 0);', _shapes())
        for (M, K, N, r, q), (kernel, bn, tn, ks, stages, tc, smem) in zip(_shapes(), got):
            what, nkb = (force, M, K, N, r, q), K // (128 if q else 64)
            limit = SMEM - (38 * 1024 if r and not tc else 0)
            if kernel == 1:
                assert M <= 32 and N <= (64 if M <= 16 else 16) * SMS and (M <= 8 or K <= 4096) and not force, what
            elif kernel == 2:
                assert 16 <= tn <= 256 and tn % 16 == 0 and 1 <= ks <= 8 and ks <= nkb and 1 <= stages <= 8, what
                assert smem <= limit - 1024 and (M + tn - 1) // tn <= 65535 and (N + 127) // 128 <= 65535, what
            else:
                assert kernel == 3 and bn in (64, 128, 192, 256) and 2 <= stages <= 8 and smem <= limit - 2560, what


def test_the_shrink_kernel_on_tcgen05_fits(plan):
    rows = [(M, K, r, n, q) for M in M_ALL for K in (64, 128, 1024, 4096, 14336) for r in (8, 16, 32, 64) for n in (1, 2, 7, 64) for q in (0, 1) if not (q and K % 128)]
    got = plan(f'ShrinkTcPlan p = plan_shrink_tc(a[0], a[1] / (a[4] ? 128 : 64), a[2], a[3], a[4], {SMS}, {SMEM}); '
               'printf("%d %d %d %d %d %d\\n", p.tn, p.ks, p.kps, p.tmem_cols, p.ring, p.smem);', rows)
    for (M, K, r, n, q), (tn, ks, kps, tmem, ring, smem) in zip(rows, got):
        what, nkb = (M, K, r, n, q), K // (128 if q else 64)
        steps = (nkb + kps - 1) // kps
        assert 16 <= tn <= 256 and tn % 16 == 0 and 1 <= ks <= 8 and steps >= ks, what                  # every block of a cluster has a slot to fill
        # whatever agents a block meets, one slot fits, and what the last MMA reads behind the lanes in use (16 KB) is inside the allocation
        whole = kps * (tn * 128 + 128 * 128 * (2 if q else 1))
        assert whole <= ring and 64 * 132 * 4 >= 16384 and smem <= SMEM - 2048, what
        assert tmem in (32, 64, 128, 256, 512) and tmem >= tn, what
        for present in (1, 2, 3, 5, 9, 17, 33, 64):                                                     # the kernel's own arithmetic
            if present > n:
                continue
            slots = 128 // r
            all_chunks = (present + slots - 1) // slots
            room = (ring // (2 * kps) - tn * 128) // (128 * 128 * (2 if q else 1))
            chunks = max(1, min(all_chunks, room, 2 if q else 4, tmem // tn))
            lane_bytes = (128 if all_chunks > 1 else present * r) * 128
            stage = kps * (tn * 128 + chunks * lane_bytes * (2 if q else 1))
            stages = min(24, ring // stage)
            assert stages >= 1 and stages * stage <= ring and chunks * tn <= tmem, (what, present)
            if (stages - 1) * stage + kps * tn * 128 + (kps - 1) * chunks * lane_bytes * (2 if q else 1) + (chunks - 1) * lane_bytes * (2 if q else 1) \
                    + (lane_bytes if q else 0) + 16384 > ring + 64 * 132 * 4:
                raise AssertionError((what, present, "the last MMA reads past the allocation"))


def test_the_small_shrink_kernel_covers_the_rows(plan):
    rows = [(M, K, most) for M in M_ALL for K in (64, 640, 4096, 14336) for most in (8, 16, 32)]
    for (M, K, most), (r, ks) in zip(rows, plan(f'ShrinkPlan p = plan_shrink(a[0], a[1], a[2], {SMS}); printf("%d %d\\n", p.rows, p.ks);', rows)):
        assert 1 <= r <= most and ks in (1, 2, 4, 8) and (ks == 1 or K // 64 >= 8 * ks), (M, K, most)
        assert (M + r - 1) // r * ks < 2 ** 31, (M, K, most)


# us of a call with agents in runs: (rows, K, N, rank, 8 bits, turn kernel, pair kernel)
MEASURED = [(64, 4096, 4096, 0, 0, 10.4, 15.8), (256, 2048, 2048, 0, 0, 8.4, 9.9), (1024, 4096, 4096, 0, 0, 29.2, 26.9), (1024, 2048, 2048, 0, 0, 14.1, 11.4),
            (512, 4096, 4096, 0, 1, 16.1, 12.3), (64, 4096, 4096, 16, 0, 13.5, 24.2), (256, 4096, 4096, 16, 0, 19.4, 24.8), (512, 4096, 4096, 16, 0, 27.4, 24.9),
            (512, 4096, 256, 16, 0, 14.0, 18.6), (2048, 4096, 4096, 64, 0, 86.0, 61.4), (256, 1024, 1024, 64, 0, 14.4, 12.1), (64, 2048, 2048, 64, 1, 14.9, 12.3),
            (64, 4096, 4096, 64, 1, 16.4, 19.8), (1024, 4096, 4096, 64, 1, 44.1, 29.2)]


def test_the_faster_main_kernel_is_taken(plan):
    got = plan(f'AdaptedPlan p = plan_adapted(a[0], a[2], a[1], a[3], a[4], {SMS}, {SMEM}, clusters); printf("%d\\n", p.kernel);', [m[:5] for m in MEASURED])
    for m, (kernel,) in zip(MEASURED, got):
        assert kernel == (2 if m[5] < m[6] else 3), m
