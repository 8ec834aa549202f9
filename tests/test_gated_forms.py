"""The forms of the gated block's kernels that the GPU tests' shapes take, by the library's own rule compiled here: every form that the rule can
choose is taken by a shape whose tiles and sums end ragged, so that a rule fitted anew cannot leave one untested.
"""
import os
import subprocess

import pytest

import test_gpu_gated
import test_gpu_gated_tiles

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2410_20650_amd", "csrc")


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    """(tokens, in_features, out_features) -> what the rule says of it."""
    exe = str(tmp_path_factory.mktemp("gated_forms") / "gated_forms")
    built = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, os.path.join(HERE, "gated_forms.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert built.returncode == 0, built.stderr

    def ask(shapes):
        told = subprocess.run([exe], input="\n".join("%d %d %d" % s for s in shapes), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in told.splitlines()]

    return ask


def taken(forms, shapes):
    """form -> the shapes (rows, columns and depth of the product, columns of a tile) that take it."""
    found = {}
    for (tokens, infeat, outfeat), (fs, fr, xs, xr, slices, ws, wr, beside) in zip(shapes, forms(shapes)):
        found.setdefault(("forward", fs, fr), []).append((tokens, outfeat, infeat, fs // 2))
        found.setdefault(("input gradient", xs, xr, slices > 1), []).append((tokens, infeat, outfeat, xs))
        found.setdefault(("weight gradients", ws, wr), []).append((outfeat, infeat, tokens, ws))
        if beside:
            found.setdefault(("both", beside > 1), []).append((tokens, infeat, outfeat, 128))
        else:
            found.setdefault(("apart", xs, ws), []).append((tokens, infeat, outfeat, xs))
    return found


def test_every_form_is_taken_ragged(forms):
    found = taken(forms, test_gpu_gated.SHAPES + test_gpu_gated_tiles.SHAPES)
    every = [("forward", 128, 2), ("forward", 128, 4), ("forward", 256, 2), ("weight gradients", 128, 2), ("weight gradients", 128, 4),
             ("weight gradients", 256, 2), ("both", False), ("both", True), ("apart", 128, 256), ("apart", 256, 128), ("apart", 256, 256)]
    every += [("input gradient", size, ring, sliced) for size, ring in ((128, 2), (128, 4), (256, 2)) for sliced in (False, True)]
    for form in every:
        ragged = [s for s in found.get(form, []) if s[0] % 64 and s[1] % s[3] and s[2] % 64]
        assert ragged, form
    # nothing else can be chosen
    assert {f[:3] for f in found if f[0] in ("forward", "weight gradients", "input gradient")} == {f[:3] for f in every if len(f) > 2 and f[0] != "apart"}


def test_tiles_of_256_end_with_little(forms):
    # a last tile of at most eight rows or columns, a last step of at most eight k, and more tiles than CUs
    found = taken(forms, test_gpu_gated_tiles.SHAPES)
    for form in (("forward", 256, 2), ("weight gradients", 256, 2), ("input gradient", 256, 2, False), ("input gradient", 256, 2, True)):
        assert any(cols % wide == 8 and 0 < depth % 64 <= 8 for rows, cols, depth, wide in found[form]), form
    assert any(rows % 256 == 1 for rows, _, _, _ in found["forward", 256, 2])
    assert any(rows % 256 == 8 for rows, _, _, _ in found["weight gradients", 256, 2])
    assert any(rows % 256 == 1 for rows, _, _, _ in found["input gradient", 256, 2, False])
    for form, halves in ((("forward", 256, 2), 1), (("weight gradients", 256, 2), 2)):
        assert any(-(-rows // 256) * -(-cols // wide) * halves > 256 for rows, cols, _, wide in found[form]), form
