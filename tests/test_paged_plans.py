"""Which kernels the steps and attentions of the GPU tests run on, on the CPU: a change of a rule must not quietly take a form out of them."""
import os
import subprocess

import pytest

from tests import paged_forms as forms

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2604_21215_amd", "csrc")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("paged_plans") / "check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "paged_plans_check.cpp"), "-o", exe], check=True)
    return lambda *a: tuple(int(v) for v in subprocess.run([exe] + [str(v) for v in a], stdout=subprocess.PIPE, text=True, check=True).stdout.split())


@pytest.mark.parametrize("form", forms.FORMS, ids=forms.NAMES)
def test_forms(ask, form):
    _, dtype, bits, d, F, most, page, _, _, pos, plan, products, tiles = form
    S = len(pos)
    assert ask("plan", most, S, d // 64, int(bool(bits))) == plan
    take, *of = ask("products", S, d, F)
    stack_engine = dtype == "bf16" and d % 256 == 0 and F % 256 == 0 and not take
    assert products == ("mm" if stack_engine else "own")
    if products == "own":
        assert of[2] == tiles
    assert max(pos) <= most + 1 and F % 8 == 0


def test_every_form_is_there(ask):
    """Parts and one part on every kind of products, both storage types and cache widths; one and four tiles of every product."""
    kinds = {(f[1], f[2], f[11], f[10][1] > 1) for f in forms.FORMS}
    for kind in (("bf16", 0, "mm"), ("bf16", 8, "mm"), ("bf16", 0, "own"), ("bf16", 8, "own"), ("f32", 0, "own"), ("f32", 8, "own")):
        assert kind + (True,) in kinds
    assert {f[10][0] for f in forms.FORMS} == {4, 16} and any(f[10][0] == 16 and f[10][1] > 1 for f in forms.FORMS)
    for dtype in ("bf16", "f32"):
        tiles = [ask("products", len(f[9]), f[3], f[4])[1:] for f in forms.FORMS if f[1] == dtype and f[11] == "own"]
        for i in range(5):
            assert {t[i] for t in tiles} == {1, 4}, (dtype, i)
    mm = [f for f in forms.FORMS if f[11] == "mm"]
    assert any(len(f[9]) <= 16 for f in mm) and any(len(f[9]) > 256 for f in mm)       # one batch tile, many
    assert any(len(f[9]) > 128 and f[3] >= 512 for f in mm) and any(-1 in f[9] for f in mm)
    for f in forms.FORMS:   # idle, empty and bounded rows wherever there is more than one
        assert len(f[9]) < 4 or (-1 in f[9] and 0 in f[9])


def test_attention_plan(ask):
    assert ask("plan", 16384, 17, 16, 0) == (16, 2)
