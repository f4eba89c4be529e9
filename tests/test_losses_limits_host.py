"""CPU checks of what the losses' calls accept, at the limits of strides, and of which rows are read through the caches."""
import os
import subprocess

import pytest

from test_losses_host import CALLS, ROOT, STRIDE, WORKSPACE, Call, losses  # noqa: F401


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("spoiled", [
    # the last element's offset in bytes is 2^63 or more: of a row far out, of a sequence far out, of both together
    dict(batch=2, length=1, stride_b=1 << 61), dict(batch=2, length=2, stride_t=1 << 60, stride_b=(1 << 60) + 100),
    dict(batch=2, length=2, grad_stride_t=1 << 61), dict(batch=2, length=1, grad_stride_b=(1 << 61) - 99)])
def test_offsets_that_no_64_bits_hold(losses, name, spoiled):
    assert Call(losses, name)(**spoiled) == STRIDE


@pytest.mark.parametrize("name", [n for n in CALLS if n != "preference_loss"])
@pytest.mark.parametrize("spoiled", [dict(stride_t=1 << 61), dict(stride_t=(1 << 61) - 99), dict(grad_stride_t=1 << 61)])
def test_offsets_of_a_single_sequence_that_no_64_bits_hold(losses, name, spoiled):
    assert Call(losses, name)(batch=1, length=2, **spoiled) == STRIDE


@pytest.mark.parametrize("field", ["stride_t", "grad_stride_t", "stride_b", "grad_stride_b"])
def test_the_largest_offsets_are_accepted(losses, field):
    # the last byte behind the last element at 2^63 - 4: refused for its workspace only, which is looked at after the strides
    shape = dict(batch=1, length=2) if field.endswith("t") else dict(batch=2, length=1)
    for name in ("token_logprobs", "policy_loss"):
        assert Call(losses, name)(**shape, **{field: (1 << 61) - 101}, workspace=None) == WORKSPACE


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("spoiled", [dict(stride_b=100, stride_t=400), dict(grad_stride_b=100, grad_stride_t=400), dict(stride_b=800 - 1)])
def test_sequences_that_interleave_are_refused_by_name(losses, name, spoiled):
    """[T, B, V] logits as [B, T, V]: rows of their own, but not one sequence behind the other."""
    status = Call(losses, name)(**spoiled)
    assert status == STRIDE and "interleave" in losses.status_string(status)
    for b, t in ((807, 101), (800, 100), (1 << 40, 1 << 20)):  # gaps of any size between rows and sequences are fine
        assert name == "token_logprobs_grad" or Call(losses, name)(stride_b=b, stride_t=t, grad_stride_b=b, grad_stride_t=t, workspace=None) == WORKSPACE


def test_rows_read_through_the_caches(tmp_path):
    """csrc/loss/loss_plan.h: all of a call's rows where the caches hold them, none of a larger one's without a mask; with one the last 600 MB,
    if what the mask keeps of them turns out to be little enough, never without asking."""
    calls = [(8, 64, 50257, 1), (8, 512, 128256, 1), (16, 1024, 32000, 1), (8, 512, 50257, 0), (4, 2, 1 << 20, 0)]
    src = tmp_path / "rows.cpp"
    src.write_text('#include <cstdio>\n#include "loss_plan.h"\nint main() { const int c[][4] = {' + ", ".join("{%d, %d, %d, %d}" % c for c in calls) +
                   '}; for (const auto& v : c) for (int masked = 0; masked < 2; ++masked) { ss_loss_params p = {v[0], v[1], v[2], v[3], 0, 0, 0, 0, 1.f, 1.f};'
                   ' const CachedRows r = cached_rows(p, (long)v[0] * v[1], masked); std::printf("%ld %d\\n", r.n, (int)r.if_sparse); } }\n')
    exe = tmp_path / "rows"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2603_16219_amd", "csrc", "loss"), "-o", exe, src], check=True)
    got = [tuple(map(int, line.split())) for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines()]
    for (B, T, V, dtype), plain, masked in zip(calls, got[::2], got[1::2]):
        rows, row = B * T, V * (2 if dtype else 4)
        if rows * row <= 1 << 28:
            assert plain == masked == (rows, 0)
        else:
            assert plain == (0, 0) and masked == (min(rows, 600_000_000 // row), 1)
