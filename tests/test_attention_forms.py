"""The forms of the attention's kernels that the GPU tests' cases take, by the library's own rule compiled here: every form that it can choose is taken by a
case, so that a rule fitted anew cannot leave one untested.
"""
import os
import subprocess

import pytest

import test_gpu_attention_forms as forms_of

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2410_20650_amd", "csrc")


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("attention_forms") / "attention_forms")
    built = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "attention_forms.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr

    def asked(calls):
        told = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in told.splitlines()]

    return asked


def taken(ask):
    """(head_dim, rows to a workgroup, waves, split or not, a step in one page or not) -> the cases."""
    found = {}
    for name, (heads, group, dim, page, window, plan) in forms_of.CASES.items():
        rows, longest = sum(n for n, _ in plan) + 5, (max((n + page - 1) // page for _, n in plan) + 1) * page
        ((tile, waves, splits),) = ask([(heads, dim, page, len(plan), heads * group, rows, window, longest)])
        found.setdefault((dim, tile, waves, splits > 1, page >= 64 if tile == 128 else None), []).append(name)
    return found


def test_every_form_is_taken(ask):
    found = taken(ask)
    kernels = {(dim, tile, waves, wide) for dim, tile, waves, _, wide in found}
    for dim in (64, 128):
        for form in ((16, 8, None), (16, 4, None), (32, 4, None), (128, 4, False), (128, 4, True)):
            assert (dim, *form) in kernels, (dim, form, found)
    assert (128, 256, 8, None) in kernels
    for tile, waves in ((16, 8), (16, 4), (32, 4), (128, 4), (256, 8)):
        for split in (False, True):
            assert any(f[1:4] == (tile, waves, split) for f in found), (tile, waves, split)


def test_the_rule(ask):
    """Any call has a form, and its splits are no more than there are keys for."""
    calls = [(h, d, p, s, h * g, r, w, n) for h in (1, 8) for d in (64, 128) for p in (16, 64) for s in (1, 48) for g in (1, 4, 17) for r in (1, 16, 500, 9000) for w in (0, 1, 300)
             for n in (16, 1000, 100000)]
    for call, (tile, waves, splits) in zip(calls, ask(calls)):
        assert (tile, waves) in ((16, 4), (16, 8), (32, 4), (128, 4), (256, 8)) and 1 <= splits <= 128
        assert splits == 1 or splits * 64 * 8 <= call[7]
        assert tile < 256 or (call[1] == 128 and call[2] >= 64)     # (the only ones that there is a kernel for)
