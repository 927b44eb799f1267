"""Which kernel a product of 8-bit rows takes: the library's planning header, compiled by itself for the host.  The GPU tests choose their
shapes for the kernels that they run; here it is held that every kernel has such a shape."""
import os
import re
import subprocess

import pytest

import test_gpu_quantized as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_12588_amd", "csrc")
QUERY = r'''
#include <cstdio>
#include "q8_plan.hpp"
int main() {
  int M, N, nk, out8, gelu;
  while (scanf("%d %d %d %d %d", &M, &N, &nk, &out8, &gelu) == 5) {
    const pab::GemmPlan g = pab::plan_q8(M, N, nk, out8, gelu);
    printf("%d %d %d %d %d\n", g.kernel, g.n_mt, g.n_nt, g.ms_tail, g.n_units);
  }
}
'''
TO_ROWS = {8, 96, 97, 113, 128, 129, 161}
TO_VALUES = {8, 9, 16, 32, 48, 64, 65, 97, 113, 128, 129, 161}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "query.cpp").write_text(QUERY)
    exe = str(d / "query")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, "-o", exe, str(d / "query.cpp")], check=True, timeout=120)

    def ask(shapes, out8, gelu=0):
        text = "".join("%d %d %d %d %d\n" % (M, N, -(-K // 128), out8, gelu) for M, N, K in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, timeout=60).stdout
        got = [tuple(int(x) for x in line.split()) for line in out.splitlines()]
        assert len(got) == len(shapes)
        return got

    return ask


def test_tested_shapes_reach_every_kernel(plan):
    for gelu in (0, 1):
        assert {g[0] for g in plan(G.SHAPES, 0, gelu)} == TO_VALUES
        assert {g[0] for g in plan(G.SHAPES, 1, gelu)} == TO_ROWS
    # large tiles: every height of a tail, alone and behind full tiles, and workgroups that go through both
    large = {(out8, g[0], g[3], g[1] > 0, g[4] > 256) for out8 in (0, 1) for g in plan(G.SHAPES, out8) if g[0] in (8, 9) and g[1] * g[2] < g[4]}
    assert {(o, k, ms, True, True) for o, k in ((0, 8), (0, 9), (1, 8)) for ms in (1, 2, 3)} <= large, large
    assert {(o, k) for o, k, _, full, _ in large if not full} == {(0, 8), (0, 9), (1, 8)}, large


@pytest.mark.parametrize("out8,kernels", [(0, TO_VALUES), (1, TO_ROWS)])
def test_every_planned_kernel_is_launched_and_covers_the_matrix(plan, out8, kernels):
    """Over a wide range of sizes the plan gives only kernels that have a launch, and as many tiles as the matrix needs."""
    sizes = sorted({int(round(1.31 ** i)) for i in range(44)})
    shapes = [(M, N, K) for M in sizes for N in (8, 64, 136, 288, 576, 1152, 3456, 4608, 13000) for K in (8, 128, 136, 576, 1152, 4608, 20000)]
    got = plan(shapes, out8)
    assert {g[0] for g in got} == kernels
    body = open(os.path.join(CSRC, "q8_api.hip")).read()
    body = body[body.index("int launch_product("):]
    assert {int(n) for n in re.findall(r"case (\d+):", body[:body.index("\n}\n")])} == TO_VALUES | TO_ROWS
    for (M, N, K), (kernel, n_mt, n_nt, ms, units) in zip(shapes, got):
        if kernel in (16, 32, 48):
            assert M <= (64 if kernel == 48 else kernel) and units * 16 >= N > (units - 1) * 16
        elif kernel in (8, 9):
            bn = 32 * kernel
            tails = units // n_nt - n_mt
            assert N >= bn and M >= 64 and K > 128 and n_nt * bn >= N > (n_nt - 1) * bn and units % n_nt == 0
            assert n_mt * 256 + tails * 64 * ms >= M and (tails == 0 or M >= 64 * ms) and (tails > 0 or ms in (0, 4) or n_mt * 256 >= M)
            assert not out8 or N % 128 == 0
        else:
            bm = {64: 64, 65: 64, 96: 64, 97: 64, 113: 96, 128: 128, 129: 128, 161: 160}[kernel]
            bn = 64 if kernel < 96 else 128
            assert n_mt * bm >= M > (n_mt - 1) * bm and n_nt * bn >= N > (n_nt - 1) * bn and units == n_mt * n_nt
            assert not kernel & 1 or units <= 256


def test_large_outputs_are_large_enough(plan):
    """... to be written past the caches, by large tiles of either width."""
    assert all(M * N * (1 if out8 else 2) > 150 << 20 for M, N, K, out8 in G.LARGE)
    assert [plan([s[:3]], int(s[3]))[0][0] for s in G.LARGE] == [8, 9, 8]


def test_few_tokens_take_their_kernel_where_it_is_faster(plan):
    """Both sides of the line as measured."""
    assert [g[0] for g in plan([(1, 6912, 1152), (3, 3256, 4440), (17, 1152, 1152)], 0)] == [16, 16, 32]
    assert not {g[0] for g in plan([(64, 1152, 4608), (20, 4608, 4608)], 0)} & {16, 32, 48}


def test_launches_have_fewer_threads_than_a_grid_holds(plan):
    """2^32 threads, workgroups of each kernel's own size counted in whole eights; matrices whose indexes would pass 2^31 have no kernel."""
    body = open(os.path.join(CSRC, "q8_api.hip")).read()
    body = body[body.index("int launch_product("):]
    threads = {int(k): int(t) for k, t in re.findall(r"case (\d+):[^;]*?dim3\((\d+)\), 0, st, p\)", body[:body.index("\n}\n")])}
    assert set(threads) == TO_VALUES | TO_ROWS
    sizes = [2**30, 2**28 * 3 + 8, 2**31 - 1024, 2**31 - 520, 200_000_000, 100_000_000, 16777216, 1_000_008]
    shapes = [(M, N, 8) for N in sizes for M in (1, 17, 64, 65, 4000)] + [(M, N, K) for M in sizes for N in (8, 136, 1152, 40000) for K in (8, 4608)]
    for out8 in (0, 1):
        got = plan(shapes, out8)
        for (M, N, K), (kernel, n_mt, n_nt, ms, units) in zip(shapes, got):
            if not kernel:
                taken = 128 * -(-K // 128) * (M + N) + M * (128 * -(-N // 128) if out8 else 2 * N)
                assert taken > 288 * 2**30 or max(M, N) > 2**31 - 1024, (M, N, K)   # only what the memory does not hold either
                continue
            assert units > 0, (M, N, K)
            groups = min(units, 256) if kernel < 16 else (units + 7) // 8 * 8
            assert groups * threads[kernel] < 2**32, (M, N, K, kernel, units)
        small = plan([(M, N, 128) for M in (1, 64, 2000) for N in range(8, 6000, 488)], out8)
        assert all(g[0] for g in small)
        assert [g[0] for g in plan([(1, 2**31 - 8, 8), (64, 2**31 - 256, 8), (2**31 - 1, 8, 8), (2**31 - 256, 4096, 256)], out8)] == [0] * 4


def test_tested_mlps_reach_every_family(plan):
    """Products of an MLP by tiles of one and of several K groups, and both by large tiles, as the largest runs do."""
    chains = [(plan([(n, F, C)], 1, 1)[0][0], plan([(n, C, F)], 0)[0][0]) for n, C, F in G.MLP_STAGES]
    assert chains[-1] == (8, 8) and {up for up, _ in chains} >= {8, 96, 97} and {down for _, down in chains} >= {8, 64, 65}, chains


def test_outputs_past_the_caches(tmp_path):
    """bf16 outputs of a tile per workgroup always, their 8-bit rows never (some wavefronts write 32 bytes of a row, and the next product reads all of
    it), large tiles' from 150 MB on; nothing whose rows do not start at multiples of 64 bytes."""
    (tmp_path / "past.cpp").write_text(r'''
#include <cstdio>
#include "q8_plan.hpp"
int main() {
  int kernel, out8; long long M, to, width, pitch;
  while (scanf("%d %d %lld %lld %lld %lld", &kernel, &out8, &M, &to, &width, &pitch) == 6)
    printf("%d\n", pab::q8_past_caches(kernel, out8, M, reinterpret_cast<void *>(to), width, pitch));
}
''')
    exe = str(tmp_path / "past")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", CSRC, "-o", exe, str(tmp_path / "past.cpp")], check=True, timeout=120)

    def ask(*rows):
        out = subprocess.run([exe], input="".join("%d %d %d %d %d %d\n" % r for r in rows), capture_output=True, text=True, check=True, timeout=60).stdout
        return [bool(int(x)) for x in out.split()]

    at = 1 << 20
    tiles = sorted((TO_ROWS | TO_VALUES) - {8, 9, 16, 32, 48})
    assert all(ask(*((k, 0, M, at, 2304, 2304) for k in tiles for M in (1, 65, 10**6))))
    assert not any(ask(*((k, 1, M, at, 1152, 1152) for k in tiles for M in (1, 65, 10**6))))
    assert ask((8, 0, 25440, at, 6912, 6912), (9, 0, 57600, at, 2304, 2304), (8, 0, 25440, at, 2304, 2304), (8, 1, 25440, at, 4608, 4608),
               (8, 1, 40000, at, 4608, 4608)) == [True, False, False, False, True]
    assert not any(ask(*((k, 0, 10**6, a, w, p) for k in tiles + [8, 9] for a, w, p in ((at + 16, 2304, 2304), (at, 2320, 2304), (at, 2304, 2320)))))
