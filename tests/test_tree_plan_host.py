"""CPU checks of what the calls with trees decide before a kernel runs: the shares of the attention's work, the pages of positions, the walk's stages
and scratch.  The headers that the kernels share are compiled by the host's compiler."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "tree_schedule.h"
#include "verify_plan.h"
int main(int argc, char** argv) {
    const auto arg = [&](int i) { return i < argc ? std::atol(argv[i]) : 0; };
    if (!std::strcmp(argv[1], "deal")) {
        const Shares s = deal((int)arg(2), (int)arg(3));
        std::printf("%d", s.shares);
        for (int w = 0; s.shares && w <= s.shares; ++w) std::printf(" %d", s.begin(w));
    } else if (!std::strcmp(argv[1], "items")) {
        const TreeItems r = tree_items(TreeTiles{(int)arg(2), (int)arg(3), (int)arg(4), 1}, (int)arg(5), (int)arg(6), arg(7) != 0, (int)arg(8));
        std::printf("%d %d %d", r.cached, r.own, r.blocks);
    } else if (!std::strcmp(argv[1], "page")) {
        const PageOf of = page_of((int)arg(2));
        for (int i = 3; i < argc; ++i) std::printf("%u ", of((unsigned)arg(i)));
    } else {
        ss_params p{};
        p.batch = (int)arg(2);
        p.k_max = (int)arg(3);
        p.vocab = (int)arg(4);
        p.dtype = (int)arg(5);
        const VerifyPlan r = verify_plan(p, (int)arg(6));
        std::printf("%d %d %d %d %d %d %d %d %d %d %zu %zu %zu %zu %zu %zu", r.stages, r.rows[0], r.rows[1], r.slices, r.slice_vecs, r.groups[0], r.groups[1],
                    r.parts, r.part_chunks, r.chunks, r.off_arrive, r.off_sums, r.off_logits, r.off_masses, r.off_best, r.bytes);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "t.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-function", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2603_16219_amd", "csrc", "tree"), "-o", at / "t", at / "t.cpp"], check=True)

    def run(*args):
        out = subprocess.run([at / "t", *map(str, args)], check=True, capture_output=True, text=True).stdout
        return [int(v) for v in out.split()]

    return run


@pytest.mark.parametrize("most", [1, 7, 256, 512, 1 << 15])
@pytest.mark.parametrize("units", [0, 1, 2, 255, 256, 511, 513, 4099, 1000003, 2**31 - 1])
def test_shares_are_equal_and_leave_nothing_out(plan, units, most):
    shares, *begin = plan("deal", units, most)
    assert shares == min(units, most)
    if shares:
        each = [b - a for a, b in zip(begin, begin[1:])]
        assert begin[0] == 0 and begin[-1] == units and min(each) >= 1 and max(each) - min(each) <= 1


@pytest.mark.parametrize("tile", [32, 64, 128])
@pytest.mark.parametrize("columns,group", [(32, 1), (64, 4), (128, 4), (256, 16)])
def test_items(plan, tile, columns, group):
    for length in (0, 1, tile - 1, tile, tile + 1, 100003, 2**31 - 1):
        for nodes in (0, 1, tile - 2, tile - 1, tile, 1024):
            up = lambda n, d: -(-n // d)
            assert plan("items", tile, columns, group, length, nodes, 0, 1024) == [up(length, tile), up(nodes + 1, tile), up((nodes + 1) * group, columns)]
    assert plan("items", tile, columns, group, -5, 7777, 1, 1024) == [0, 1, -(-1025 * group // columns)]  # a marked sequence: all its rows, and one tile


def test_pages_of_positions(plan):
    for size in (1, 2, 3, 5, 7, 16, 24, 100, 127, 128, 129, 1000, 4095, 4096, 4097, 65535, 65537, 99962, 2**30 - 1, 2**30, 2**30 + 1, 2**31 - 1):
        last = 2**31 - 1
        at = sorted({p for k in (0, 1, 2, 3, 1000, last // size // 2, last // size - 1, last // size) for p in (k * size - 1, k * size, k * size + 1) if 0 <= p <= last}
                    | {0, last - 1, last})
        assert plan("page", size, *at) == [p // size for p in at], size


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V", [1, 7, 9, 513, 32000, 50257, 128256, 151936, 1 << 20])
@pytest.mark.parametrize("N", [0, 1, 2, 7, 63, 64, 1024])
def test_walk_s_stages_and_scratch(plan, N, V, dtype):
    for B in (1, 2, 64, 1000):
        if B * (N + 1) > 1 << 20:
            continue
        for units in (1, 256):
            stages, r0, r1, slices, vecs_each, g0, g1, parts, chunks_each, chunks, *off, total = plan("walk", B, N, V, dtype, units)
            vecs, lanes = V // (8 if dtype == 1 else 4), 256
            assert 0 <= stages <= 2 and (stages == 0) == (N == 0)
            if stages:
                assert [r0, r1][stages - 1] >= N + 1 and min([r0, r1][:stages]) >= 1 and all(1 <= g <= N + 1 for g in [g0, g1][:stages])
            assert 1 <= slices <= 16 and slices * vecs_each >= vecs
            assert 1 <= parts <= 32 and parts * chunks_each >= chunks and (chunks - 1) * lanes >= vecs and chunks <= 1025
            need = [B * 16 * (stages + 1), B * 256 if parts > 1 else 0, B * (N + 1) * 2 * slices * 16, B * N * 8, B * chunks * 8, B * parts * 16]
            start = [0, *off]
            assert all(s % 16 == 0 for s in start)
            assert all(s + n <= e for s, n, e in zip(start, need, [*off, total]))
