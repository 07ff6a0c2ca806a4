"""The parameter update of the Muon step on the GPU against the fp64 oracle, with parameters of the size of the update, so that every term of it
counts: results that leave one out, or have its sign wrong, are shown to lie outside the tolerance.

Tolerance: X is rounded once to its type, half a step of every entry; lr scale O is as far off as O is (test_gpu_muon.py), in the norm
and 8 times that for an entry, relative to itself or the rms of all; 1 - lr wd and lr scale are rounded to fp32 and so is their
difference, 2^-22 of both terms."""
import math

import numpy as np
import pytest

from oracle.optimizers_oracle import muon_step
from paper_2605_16341_amd import binding
from test_gpu_muon import HALF, QUINTIC, matrix, tolerance, types, upload

pytestmark = pytest.mark.gpu

LR, DECAY, MU = 0.5, 1.0, 0.8
SHAPES = [(8 + 5 * i, 90 - 4 * i) for i in range(20)] + [(64, 96)] * 3 + [(1, 33), (33, 1), (7, 1), (1, 1), (200, 130), (130, 200), (300, 1100), (1100, 300)]
RULES = {"none": lambda m, n: 1.0, "spectral": lambda m, n: math.sqrt(max(1.0, m / n)), "rms": lambda m, n: 0.2 * math.sqrt(max(m, n))}


class Expected:
    """X, M after a step in fp64, and whether another X is within the tolerance."""

    def __init__(self, x, g, m, scale, nesterov, fast, storage):
        self.x, self.m, self.o = muon_step(x, g, m, QUINTIC, MU, LR, DECAY, scale, nesterov)
        self.before, self.scale, self.storage = x, scale, storage
        self.tol = tolerance(g + MU * self.m if nesterov else self.m, QUINTIC, not fast, "f32")
        self.room = LR * scale * self.tol

    def misses(self, got):
        """By how much `got` leaves the tolerance: at most 1 is within."""
        exact = 2.0 ** -22 * (np.abs(self.before) + LR * self.scale * np.abs(self.o))
        rms = np.linalg.norm(self.o) / math.sqrt(self.o.size)
        entry = self.storage * np.abs(self.x) + exact + 8 * self.room * np.maximum(np.abs(self.o), rms)
        off = np.abs(got - self.x)
        return max(np.max(off / entry), np.linalg.norm(off) / (self.storage * np.linalg.norm(self.x) + np.linalg.norm(exact) + self.room * np.linalg.norm(self.o)))

    def wrong_ones(self, other_nesterov):
        """What X would be with a part of the formula missing."""
        step = LR * self.scale * self.o
        keep = (1 - LR * DECAY) * self.before
        yield "untouched", self.before
        yield "decay only", keep
        yield "sign of O", keep + step
        yield "no decay", self.before - step
        yield "sign of the decay", (1 + LR * DECAY) * self.before - step
        if abs(self.scale - 1) > 0.3:
            yield "no scale", keep - LR * self.o
        if np.linalg.norm(other_nesterov - self.o) > 0.3 * np.linalg.norm(self.o):
            yield "the other momentum", keep - LR * self.scale * other_nesterov


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("scale", ["none", "spectral", "rms"])
@pytest.mark.parametrize("x,g,precision", [("bf16", "bf16", "auto"), ("f32", "f32", "auto"), ("f32", "bf16", "fast"), ("bf16", "f32", "auto"), ("bf16", "f32", "fast")])
def test_every_term_of_the_update(x, g, precision, scale, nesterov):
    import torch
    rng = np.random.default_rng(21)
    opt = binding.Muon(SHAPES, x_dtype=x, g_dtype=g, precision=precision, lr=LR, weight_decay=DECAY, mu=MU, nesterov=nesterov, scale=scale)
    # entries of the update: O has singular values around 1
    size = [LR * RULES[scale](m, n) * math.sqrt(min(m, n) / (m * n)) for m, n in SHAPES]
    X = [upload(torch, r * rng.standard_normal(s), types(torch, x))[1] for s, r in zip(SHAPES, size)]
    M = [upload(torch, matrix(rng, *s), torch.float32)[1] for s in SHAPES]
    fast = precision == "fast" or x == g == "bf16"
    told_apart = set()
    for step in range(2):
        G = [upload(torch, matrix(rng, *s), types(torch, g))[1] for s in SHAPES]
        before = [[t.double().cpu().numpy() for t in seq] for seq in (X, G, M)]
        opt.step(X, G, M)
        assert opt.info() == [0] * len(SHAPES)
        for i, s in enumerate(SHAPES):
            args = [seq[i] for seq in before] + [float(np.float32(RULES[scale](*s)))]
            want = Expected(*args, nesterov, fast, HALF[x])
            assert np.allclose(M[i].double().cpu().numpy(), want.m, rtol=2.0 ** -22, atol=2.0 ** -22 * np.abs(want.m).max())
            assert want.misses(X[i].double().cpu().numpy()) <= 1, (step, s)
            other = Expected(*args, not nesterov, fast, HALF[x]).o
            for name, wrong in want.wrong_ones(other):
                assert want.misses(wrong) > 1, (name, s)
                told_apart.add(name)
    assert told_apart >= {"untouched", "decay only", "sign of O", "no decay", "sign of the decay", "the other momentum"}
    assert scale == "none" or "no scale" in told_apart
