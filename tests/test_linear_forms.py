"""Which kernels the calls around the quantized linear layer launch, asked of the rules themselves (csrc/wq_linear_form.h) on the
CPU: the GPU tests' sizes choose the instances that they are there for, and together they reach every one."""
import itertools
import os
import subprocess

import pytest

import test_linear_block_gpu as block
import test_linear_forms_gpu as forms
import test_linear_values_gpu as values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = tmp_path_factory.mktemp("form") / "form"
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2412_19867_amd", "csrc"),
                    os.path.join(ROOT, "tests", "linear_form_check.cpp"), "-o", str(exe)], check=True)

    def run(questions):
        text = "\n".join(" ".join(str(int(v)) if k else v for k, v in enumerate(q)) for q in questions)
        return subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    return run


def product_cases():
    """(what is launched according to the table or None, group size, gated, question) of the tests with 8-bit and 4-bit weights"""
    for n, couts, cins, want in forms.PRODUCTS.values():
        for g, (gated, Cout) in itertools.product(cins, zip((True, False), couts)):
            yield want, g, gated, ("product", n, cins[g], Cout, g, gated)
    for n, Cout, long_k in block.FORMS.values():
        for g, gated in itertools.product(block.SHORT, (True, False)):
            yield None, g, gated, ("product", n, 2048 if long_k and g >= 128 else block.SHORT[g], Cout if gated else Cout - 3, g, gated)
    for n, _, Cin, Cout, g, _, gated, _ in block.PRODUCTS:
        yield None, g, gated, ("product", n, Cin, Cout, g, gated)


def test_product_cases_take_the_forms_that_they_name(ask):
    cases = [c for c in product_cases() if c[0]]
    for (want, *_, question), got in zip(cases, ask([c[3] for c in cases])):
        assert got == want, question


@pytest.mark.parametrize("layer,waves", [((1, 5120, 27648, 128, 1), 4), ((1, 8192, 28672, 128, 1), 4), ((2, 4096, 16384, 128, 0), 4),
                                         ((1, 4096, 14336, 128, 0), 4), ((4, 2048, 12288, 128, 0), 4), ((1, 8192, 8192, 128, 0), 8),
                                         ((2, 2048, 8192, 64, 0), 8), ((1, 4096, 4096, 128, 0), 8), ((1, 2048, 4096, 64, 0), 8)])
def test_waves_of_one_launch_follow_the_measured_side(ask, layer, waves):
    """Layers whose two sides were measured."""
    assert ask([("product", *layer)])[0].split(",")[0] == f"rows1 x{waves} itself"


@pytest.mark.parametrize("layer,launches", [((4, 4096, 4096, 128, 0), 2), ((24, 1024, 1024, 64, 0), 2), ((8, 2048, 2048, 128, 0), 2),
                                            ((1, 16384, 4096, 128, 0), 2), ((1, 8192, 4096, 128, 0), 1), ((3, 4096, 4096, 128, 0), 1),
                                            ((60, 512, 800, 256, 0), 1)])
def test_a_graph_gets_the_form_that_takes_less_of_the_cards_time(ask, layer, launches):
    """Layers whose two sides were measured in a graph; launched one by one, where a launch costs the host more, all take one."""
    assert ask([("captured", *layer)])[0].split(",")[0].endswith("itself") == (launches == 1)
    assert ask([("product", *layer)])[0].split(",")[0].endswith("itself")


def test_the_long_sums_take_the_forms_that_they_name(ask):
    want = {"rows": "rows1 x4", "rows2": "rows2 x4", "teams4": "tiles64 4", "teams2": "tiles64 2", "teams1": "tiles64 1", "large": "tiles128"}
    got = ask([("product", n, 8192, Cout, 32, False) for n, Cout in values.LONG.values()])
    assert {k: v.split(", ")[0] for k, v in zip(values.LONG, got)} == want


def test_every_product_kernel_is_reached(ask):
    """Forms of the product x group sizes (256 and 512 share their code, but not how a group ends) x gated; each with both widths."""
    cases = list(product_cases())
    reached = set()
    for (_, g, gated, _), got in zip(cases, ask([c[3] for c in cases])):
        reached |= {(form, g, gated) for form in got.split(", ")}
    every = set(itertools.product(("rows1 x8 itself", "rows1 x4 itself", "rows1 x4", "rows2 x4", "tiles64 4", "tiles64 2", "tiles64 1", "tiles128"),
                                  (32, 64, 128, 256, 512), (True, False)))
    assert reached == every, (every - reached, reached - every)


def test_every_quantizer_is_reached(ask):
    norm = block.NORMS + forms.WIDE
    got = set(ask([("quantize", n, C, True, True) for n, _, C, _ in norm]))
    assert {tuple(map(int, f.split()[1:])) for f in got if f != "row"} == {(w, 1, 1) for w in (1, 2, 4, 8)} | {(8, v, 1) for v in (2, 4, 8)}
    assert "row" in got
    assert set(ask([("quantize", n, C, True, True) for n, _, C, _ in forms.WIDE])) == {"pieces 8 8 1"}
    many = {(f, g) for (n, _, C, g), f in zip(forms.MANY, ask([("quantize", n, C, False, True) for n, _, C, _ in forms.MANY]))}
    assert many == {("pieces 1 1 2", g) for g in (32, 64, 128, 256, 512)}
    few = {(f, g) for (n, _, C, g), f in zip(block.NORMS, ask([("quantize", n, C, False, True) for n, _, C, _ in block.NORMS]))}
    assert few == {("pieces 1 1 1", g) for g in (32, 64, 128, 256, 512)}
