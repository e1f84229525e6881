"""How weight gradients are split, and that the exact cases see what a wrong split would do (no GPU needed)."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from weight_grad_cases import CASES, CODES, gradients, inputs, three_parts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2006_02924_amd", "csrc")


@pytest.fixture(scope="module")
def split_of(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path_factory.mktemp("split") / "weight_split"
    subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "weight_split.cpp"), os.path.join(CSRC, "adasum_weight_split.cpp"), "-o", str(exe)],
                   check=True)

    def ask(shapes):
        lines = "".join("%d %d %d %d\n" % s for s in shapes)
        out = subprocess.run([str(exe)], input=lines, capture_output=True, text=True, check=True, timeout=60).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return ask


def test_the_exact_cases_have_the_squares_and_parts_that_they_are_meant_for(lib, split_of):
    shapes = [(n, width, outputs, CODES[dtype]) for dtype, _, n, outputs, width, _, _ in CASES]
    for case, shape, (edge, parts, steps, total) in zip(CASES, shapes, split_of(shapes)):
        assert (edge, parts) == case[5:], case
        need = C.c_size_t(0)
        assert lib.adasum_checkpoint_weight_grad_workspace_bytes(*shape, C.byref(need)) == 0 and need.value == total
    # every kind of square is there for every type, with parts and without
    for dtype in CODES:
        for ragged in (False, True):
            for edge in (128, 256):
                assert any(c[0] == dtype and c[5] == edge and (c[3] % 8 != 0) == ragged for c in CASES)
        assert {c[1] for c in CASES if c[0] == dtype and c[5:] == (256, 1)} == set(CODES)
        for joined in (False, True):
            assert any(c[0] == dtype and c[5] == 256 and (c[6] > 1) == joined and c[3] % 8 == 0 for c in CASES)


def test_parts_cover_every_step_once(split_of):
    shapes = [(n, width, outputs, code) for n in (0, 1, 31, 32, 33, 64, 65, 1000, 4093, 16400, 40000, 1 << 20, (1 << 31) - 65536)
              for outputs, width in ((1, 1), (64, 64), (1000, 2048), (1024, 1024), (4096, 4096)) for code in CODES.values()]
    for (n, _, _, code), (edge, parts, steps, _) in zip(shapes, split_of(shapes)):
        step = 32 if code == 0 else 64
        assert edge in (128, 256) and parts >= 1
        assert parts * steps * step >= n and (n == 0 or (parts - 1) * steps * step < n)


def small(dtype):
    return (dtype, "f32", 300, 24, 40)


@pytest.mark.parametrize("dtype", list(CODES))
def test_a_lost_or_doubled_token_shows(dtype):
    """The mistake is made here, in what the result would be."""
    dy, x = inputs(small(dtype), "whole", "cpu")
    nothing = torch.zeros(24, 40), torch.zeros(24)
    want = gradients(dy, x, *nothing, torch.float32)
    for t in (0, 63, 64, 127, 128, 299):
        for times in (0.0, 2.0):
            wrong = dy.clone()
            wrong[t] *= times
            weight, bias = gradients(wrong, x, *nothing, torch.float32)
            assert (weight != want[0]).all() and (bias != want[1]).all()
    # two tokens of dy exchanged
    swapped = dy.clone()
    swapped[[17, 81]] = dy[[81, 17]]
    assert (gradients(swapped, x, *nothing, torch.float32)[0] != want[0]).any()


def test_a_lost_part_of_fp32_shows():
    dy, x = inputs(small("f32"), "three parts", "cpu")
    nothing = torch.zeros(24, 40), torch.zeros(24)
    want = gradients(dy, x, *nothing, torch.float32)
    first = dy.bfloat16().float()
    second = (dy - first).bfloat16().float()
    third = dy - first - second
    assert (second != 0).any() and (third != 0).any() and torch.equal(third.bfloat16().float(), third)
    for wrong in (first, first + second, first + third):
        weight, bias = gradients(wrong, x, *nothing, torch.float32)
        assert (weight != want[0]).float().mean() > 0.5 and (bias != want[1]).float().mean() > 0.5
    dy, _ = three_parts(9000, 1024, 8, 1, "cpu")
    assert (dy != 0).any(1).all() and int((dy != 0).sum(0).max()) <= 40
