"""Which kernels the rules of csrc/wq_fp8_form.h choose: every one of them is reached by sizes that the GPU tests run."""
import os
import subprocess

import pytest

import test_fp8_gpu as t
import test_fp8_forms_gpu as big

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("form") / "check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2412_19867_amd", "csrc"),
                    os.path.join(ROOT, "tests", "fp8_form_check.cpp"), "-o", exe], check=True)

    def f(lines):
        out = subprocess.run([exe], input="\n".join(" ".join(map(str, line)) for line in lines) + "\n", text=True, capture_output=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return f


def groups(n):
    return -(-n // 128)


def test_the_sizes_of_the_form_tests_reach_their_forms(ask):
    for name, (rows, C, O, gated) in big.FORWARD.items():
        got = ask([("f", rows, O // 2 if gated else O, int(gated), groups(C), 1)])[0]
        assert (got[0], got[1]) == (0, big.TILES[name.split("-")[0]]), name
    for name, (rows, C, O) in big.INPUT_GRADS.items():
        for exact in (0, 1):
            want = big.TILES[name.split("-")[0]]
            got = ask([("f", rows, C, 0, groups(O), exact)])[0]
            assert got[0] == 0 and (got[1] == want or exact), name
    for name, (rows, C, O) in big.WEIGHT_GRADS.items():
        assert ask([("g", O, C, groups(rows))])[0][0] == big.TILES[name], name
    assert {n.split("-")[0] for n in big.FORWARD} == set(big.TILES)
    # four teams are for exact sums, and no gradient of weights takes two of 128
    assert set(big.INPUT_GRADS) == set(big.TILES) - {"t64four"} and set(big.WEIGHT_GRADS) == set(big.TILES) - {"t64four", "t128two"}
    for rows in (17, 200, 500, 2000):
        for outs in (40, 300, 2000):
            for g in (1, 15, 16, 80):
                assert ask([("f", rows, outs, 0, g, 0)])[0][1] != 5 and ask([("g", rows, outs, g)])[0][0] not in (5, 7)


def test_few_rows_reach_every_kernel_for_them(ask):
    seen = set()
    for n, C, O, gated in [(n, C, O, gated) for n, _, C, O, _, gated, _ in t.PRODUCTS] + big.FEW:
        blocks, _, takes, captured, waves = ask([("f", n, O // 2 if gated else O, int(gated), groups(C), 1)])[0]
        if blocks:
            seen.add((gated, blocks, bool(takes)))
            if takes:
                seen.add((gated, "waves", waves))
    for gated in (False, True):
        assert {(gated, 1, True), (gated, 1, False), (gated, 2, False), (gated, "waves", 4), (gated, "waves", 8)} <= seen, {(gated, 1, True), (gated, 1, False), (gated, 2, False), (gated, "waves", 4), (gated, "waves", 8)} - seen


def test_lines_of_the_rules(ask):
    """A size on either side of each line."""
    tile = lambda rows, outs, g, exact=1: ask([("f", rows, outs, 0, g, exact)])[0][:2]   # noqa: E731
    assert tile(128, 1792, 8) == (2, 0) and tile(129, 1792, 8)[0] == 0 and tile(128, 1824, 8)[0] == 0
    assert tile(16, 14400, 8) == (1, 0) and tile(17, 2048, 8) == (1, 0) and tile(17, 2064, 8) == (2, 0)
    assert tile(4096, 4096, 16)[1] == 0 and tile(4096, 4096, 15)[1] == 1
    assert tile(1024, 1024, 16)[1] == 5 and tile(1024, 1024, 15)[1] == 6 == tile(1024, 1024, 16, 0)[1] and tile(1025, 1024, 16)[1] == 4
    assert tile(2049, 1024, 15)[1] == 3 and tile(2048, 1024, 15)[1] == 4 and tile(2048, 1024, 6)[1] == 3
    assert tile(2048, 2048, 16)[1] == 7 and tile(2048, 2048, 15)[1] == 3 and tile(2048, 2048, 39, 0)[1] == 2 and tile(2048, 2048, 40, 0)[1] == 7
    assert tile(2048, 2049, 17)[1] == 3 and tile(2048, 2049, 18)[1] == 2 and tile(2048, 2049, 28, 0)[1] == 1
    assert tile(2048, 3104, 9)[1] == 1 and tile(2048, 3104, 8)[1] == 3
    assert tile(1, 1, 1) == (1, 0)
    # captured streams quantize x in the same launch up to 12288 elements, others up to 16384
    f = lambda rows, g: ask([("f", rows, 1024, 0, g, 1)])[0][2:4]   # noqa: E731
    assert f(1, 96) == (1, 1) and f(1, 97) == (1, 0) and f(1, 128) == (1, 0) and f(1, 129) == (0, 0) and f(16, 6) == (1, 1) and f(16, 9) == (0, 0)
