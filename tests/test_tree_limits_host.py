"""CPU checks of positions and pages at the ends of 32 bits, with the headers that the kernels share, compiled for the host with its checks of overflows;
and of the refusal of outputs that are inputs."""
import os
import subprocess

import pytest
import torch

from test_tree_host import AT, PARAM, call, tree  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include "tree_schedule.h"
int main(int argc, char** argv) {
    const auto arg = [&](int i) { return (int)std::atol(argv[i]); };
    if (argc == 7) {
        const TablePiece r = table_piece(arg(1), arg(2), page_of(arg(3)), arg(3), arg(4), arg(5), arg(6));
        std::printf("%d %d %d", r.from, r.entries, r.until);
    } else {
        const PageRange r = pages_written(arg(1), arg(2), arg(3));
        std::printf("%d %d", r.first, r.more);
    }
    return 0;
}
"""
MOST, LAST = 1024, 2**31 - 1
PAGES = [1, 2, 3, 16, 1000, 2**30, LAST]


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("limits")
    (at / "t.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-Wno-unused-function", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2603_16219_amd", "csrc", "tree"), "-o", at / "t", at / "t.cpp"], check=True)
    return lambda *args: [int(v) for v in subprocess.run([at / "t", *map(str, args)], check=True, capture_output=True, text=True).stdout.split()]


@pytest.mark.parametrize("page", PAGES)
@pytest.mark.parametrize("tile", [64, 128])
def test_pieces_of_the_table(program, tile, page):
    for length in (1, tile, tile + 1, 5000, LAST - tile, LAST - 1, LAST):
        cached = -(-length // tile)
        for t in sorted({0, cached // 2, max(0, cached - 17), max(0, cached - 9), cached - 1}):
            start, entries, until = program(t, tile, page, length, cached, MOST)
            last = (length - 1) // page
            assert start == t * tile // page and 1 <= entries <= MOST and start + entries - 1 <= last
            assert t < until <= cached and until == min(cached, t + ((start + MOST) * page - t * tile) // tile)
            assert (min(length, until * tile) - 1) // page < start + entries  # the pages of all its tiles are there


@pytest.mark.parametrize("page", PAGES)
def test_pages_that_a_commit_writes(program, page):
    for length in (0, 1, 999, LAST - 1025, LAST - 300, LAST - 2, LAST - 1):
        for rows in (0, 1, 255, 256, 1024):
            if length + rows + 1 <= LAST:
                assert program(length, rows, page) == [length // page, (length + rows) // page - length // page]


@pytest.mark.parametrize("name,arrays", [
    *[("commit", ("new_len", k)) for k in ("cache_len", "accepted_len", "path", "block_table")],
    *[("verify", (o, i)) for o in ("accepted_len", "path", "next_token", "next_token_logprob") for i in ("tokens", "parents", "tree_len", "uniforms")],
    ("verify", ("accepted_len", "next_token")), ("verify", ("path", "accepted_len")), ("verify", ("next_token_logprob", "next_token"))])
def test_no_output_is_an_input_or_another_output(tree, name, arrays):
    assert call(tree, name, **{k: AT for k in arrays}) == PARAM


def test_numbers_beyond_32_bits_are_out_of_range(tree):
    t = torch.tensor([0, -1, 5, 2**31 - 1, 1 - 2**31, -2**31, 2**31, 2**32 + 5, -2**32 + 5, 2**63 - 1, -2**63])
    low = -2**31
    assert tree._ints(t, "t", (11,), t.device).tolist() == [0, -1, 5, 2**31 - 1, 1 - 2**31, low, low, low, low, low, low]
