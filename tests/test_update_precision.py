"""CPU-only: the bounds that the updates are held to (update_precision.py) see a low part that is lost anywhere."""
import pytest
import torch

import training_reference as ref
import update_precision as up

SIZES = [(16, 16), (17, 16), (60, 40), (64, 384), (96, 224), (128, 128), (130, 200), (200, 333), (250, 250), (257, 259),
         (517, 200), (500, 380), (640, 640)]


@pytest.mark.parametrize("r,c", SIZES)
@pytest.mark.parametrize("kind,steps", [("strong", 1), ("strong", 2), ("plain", 5), ("mixed", 5), ("strong", 5)])
def test_lost_parts_are_seen(r, c, kind, steps):
    """(Of few steps where singular values are large: the powers of small ones add little.  There the loss of one of
    two operands that are the same matrix mostly falls into directions that the step does not raise.)"""
    g = up.matrix(r, c, r + c, kind)
    coefs = (ref.MUON,) * steps
    want = up.expected(g, coefs=coefs)
    x = up.start(g, dtype=torch.float32)
    shape = (lambda y: y.t()) if r >= c else (lambda y: y)
    up.check(shape(up.emulated(x, coefs)), want)
    either = ("left", "right")
    losses = [dict(gram=either), dict(poly=either), dict(apply=("left",)), dict(apply=("right",)),
              dict(gram=either, poly=either, apply=either)]
    if steps == 5:
        losses += [dict(gram=("left",)), dict(gram=("right",)), dict(poly=("left",)), dict(poly=("right",))]
    for lost in losses:
        got = shape(up.emulated(x, coefs, **lost))
        out, entries, norm = want
        off = (got.double() - out).abs()
        assert bool((off > entries).any()) and float(off.norm()) > norm, (lost, float((off / entries).max()), float(off.norm()) / norm)


@pytest.mark.parametrize("r,c", SIZES)
@pytest.mark.parametrize("kind", ["plain", "mixed"])
def test_a_wrong_entry_is_seen(r, c, kind):
    """One entry off by a ten-thousandth of the largest."""
    g = up.matrix(r, c, 1, kind)
    out, entries, _ = up.expected(g)
    assert float(entries.max()) < 1e-4 * float(out.abs().max())
