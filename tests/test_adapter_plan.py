"""The rules by which calls of the adapters are shared out (csrc/adapter_plan.h), compiled for the host: the cases that GPU tests compare with the
oracle have the tiles, slices, rounds and pieces for which they are there."""
import os
import shutil
import subprocess

import pytest

import adapter_cases as C

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2505_03803_amd", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    exe = str(tmp_path_factory.mktemp("plan") / "check")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-I", CSRC, "-o", exe, os.path.join(HERE, "host", "adapter_plan_check.cpp")], check=True)

    def of(seqs, tokens, n, rank, depth, wide, mats, offsets=True, drop=False, wide_y=False):
        line = " ".join(str(int(v)) for v in (seqs, tokens, n, rank, offsets, drop, mats, depth, wide, wide_y))
        return tuple(map(int, subprocess.run([exe], input=line, capture_output=True, text=True, timeout=60, check=True).stdout.split()))

    return of


@pytest.mark.parametrize("case,cut", C.SUMS, ids=lambda c: str(c))
def test_pieces(plan, case, cut):
    lens, _, n, rank, K, N, mats = case
    for drop in (False, True):
        assert plan(len(lens), sum(lens), n, rank, N, K, mats, drop=drop)[3] == cut
        assert plan(len(lens), sum(lens) + 3, n, rank, N, K, mats, drop=drop)[3] == cut          # rows of no sequence
    assert max(lens) % cut % 32 != 0


@pytest.mark.parametrize("case,rows,slices,rounds", C.ROUNDS, ids=lambda c: str(c))
def test_rounds(plan, case, rows, slices, rounds):
    lens, _, n, rank = case
    for drop in (False, True):
        for wide_y in (False, True):
            assert plan(len(lens), sum(lens) + 3, n, rank, C.NARROW, C.WIDE, 8, drop=drop, wide_y=wide_y)[:3] == (rows, slices, rounds)


@pytest.mark.parametrize("case,rounds", C.GATHERED, ids=lambda c: str(c))
def test_rounds_of_single_tokens(plan, case, rounds):
    tokens, n, rank = case
    assert plan(tokens, tokens, n, rank, C.NARROW, C.WIDE, 8, offsets=False)[:3] == (16, 1, rounds)


@pytest.mark.parametrize("case,rows,slices,rounds", C.SLICES, ids=lambda c: str(c))
def test_slices(plan, case, rows, slices, rounds):
    lens, _, n, rank, K, N, mats = case
    for wide_y in (False, True):
        assert plan(len(lens), sum(lens) + 3, n, rank, K, N, mats, wide_y=wide_y)[:3] == (rows, slices, rounds)


def test_plans_are_of_the_kinds_that_there_are(plan):
    for rank in (8, 24, 64, 128):
        for tokens in (1, 40, 333, 2048, 8192):
            for wide in (8, 264, 4096, 14336):
                rows, slices, rounds, cut = plan(1, tokens, 1, rank, 4096, wide, 1)
                assert rows in (16, 32) and 1 <= slices <= -(-wide // 64) and rounds >= 1 and cut in (64, 128, 256, 512, 1024, 2048, 4096)
