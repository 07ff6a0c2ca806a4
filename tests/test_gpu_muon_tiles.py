"""Muon on the GPU at sizes that reach every tile width of every product, against the fp64 oracle and, in one word, against the same
matrices on other tiles.

The matrices are block diagonal under random permutations of their rows and columns: every tile holds entries of every block and
zeros between them, and the oracle iterates on the blocks.

Tolerance of O: in two words as derived in test_gpu_muon.py, from the singular values of all blocks (1e-5: a single wrong entry of S is
far beyond it).  In one word that sum of largest errors is 2e-2, which a few wrong entries would pass.  The roundings are independent and
of rms 0.4 u, so their squares add up: `spread`, of which 3 times is allowed in the norm and 8 times for an entry, relative to itself
and the rms of entries (5.5 deviations are the largest of 16 million).

On other tiles, every entry of a product is the same sum of the same words in the same order, k by k: the same bits, where matrices go
step by step.  Of steps that share a Gram matrix, P S and (P S) P are not quite symmetric once their factors are rounded, and which of
their entries are computed and which mirrored goes by the tile: there both are off by their spread, sqrt(2) of it between them."""
import math

import numpy as np
import pytest

from muon_sets import ONE_WORD_PAIRS, ONE_WORD_SINGLES, TWO_WORDS, shapes_of
from paper_2605_16341_amd import binding
from test_gpu_muon import HALF, check

pytestmark = pytest.mark.gpu

QUINTIC = binding.MUON_COEFFS


def scattered(rng, m, n):
    """(matrix, [(rows, columns)] of its blocks)"""
    blocks = max(2, min(m, n) // 400)
    rows, cols = np.array_split(rng.permutation(m), blocks), np.array_split(rng.permutation(n), blocks)
    a = np.zeros((m, n), dtype=np.float32)
    for r, c in zip(rows, cols):
        a[np.ix_(r, c)] = 1e-2 * rng.standard_normal((len(r), len(c)))
    return a, list(zip(rows, cols))


def iterate(a, blocks):
    """(O, singular values of X_0) in fp64"""
    norm = np.sqrt(np.sum(a.astype(np.float64) ** 2)) + 1e-7
    out, spectrum = np.zeros(a.shape), np.zeros(min(a.shape))
    at = 0
    for r, c in blocks:
        x = a[np.ix_(r, c)].astype(np.float64) / norm
        s = np.linalg.svd(x, compute_uv=False)
        spectrum[at:at + len(s)] = s
        at += len(s)
        for ca, cb, cc in QUINTIC:
            gram = x @ x.T
            x = ca * x + (cb * gram + cc * gram @ gram) @ x
        out[np.ix_(r, c)] = x
    return out, spectrum


def tolerance(s, longest, exact):
    """(sum of the largest errors, root of the sum of squares of those to expect) relative to O, in the norm"""
    u = 2.0 ** -11 if not exact else 2.0 ** -22 + 2.0 ** -24 * (1 + math.sqrt(longest / 16))
    values = [s]
    for ca, cb, cc in QUINTIC:
        s = ca * s + cb * s ** 3 + cc * s ** 5
        values.append(s)
    total, squares, grow, slope = 0.0, 0.0, np.ones_like(s), np.ones_like(s)
    for (ca, cb, cc), v in zip(reversed(QUINTIC), reversed(values[:-1])):
        grow = grow * np.abs(ca + cb * v ** 2 + cc * v ** 4)
        slope = slope * np.abs(ca + 3 * cb * v ** 2 + 5 * cc * v ** 4)
        one = np.linalg.norm(v) * math.sqrt(np.mean(np.maximum(grow, slope) ** 2))
        total += 3 * u * one
        squares += 3 * (0.4 * u * one) ** 2
    norm = np.linalg.norm(values[-1])
    return total / norm, math.sqrt(squares) / norm


def buffers(torch, groups, dtype, seed):
    """Device matrices of a set, and {index: (host matrix, blocks)} of the first and last of each group; matrices of the same group, place
    and seed are the same in every set."""
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    out, known = [], {}
    for g, (count, m, n) in enumerate(groups):
        for k in range(count):
            if k in (0, count - 1):
                a, blocks = scattered(np.random.default_rng((seed, g, k > 0)), m, n)
                t = torch.from_numpy(a).to("cuda:0", dtype)
                known[len(out)] = (t.float().cpu().numpy(), blocks)
                out.append(t)
            else:
                out.append((1e-2 * torch.randn(m, n, device="cuda:0", generator=gen)).to(dtype))
    return out, known


def orthogonalised(torch, groups, g, precision, seed):
    """O in fp32 of the orthogonalisation, X = O of a step from zero, in bf16 where the precision is fast; and the matrices known"""
    shapes = shapes_of(groups)
    A, known = buffers(torch, groups, torch.bfloat16 if g == "bf16" else torch.float32, seed)
    opt = binding.Muon(shapes, x_dtype="f32", g_dtype=g, precision=precision)
    O = [torch.full(s, 7.0, device="cuda:0") for s in shapes]
    opt.orthogonalise(A, O)
    step = binding.Muon(shapes, x_dtype=g, precision=precision, mu=0.0, lr=-1.0, scale="none")
    X, M = [torch.zeros_like(a) for a in A], [torch.zeros(s, device="cuda:0") for s in shapes]
    step.step(X, A, M)
    assert opt.info() == step.info() == [0] * len(shapes)
    return O, X, known


def name_of(groups):
    return "+".join("%dx%dx%d" % g for g in groups)


def close(got, want, spread, storage):
    """Within `spread` as described above, and half a step of the storage type of every entry (once for each of two stored matrices).
    Outside the blocks there are only zeros to add up; errors lie within them, with the rms of the entries there: of b blocks of a
    matrix's b^2, sqrt(b) times that over the whole matrix."""
    off, want = (got.double() - want).abs(), want.abs()
    assert bool((got[want == 0] == 0).all())
    rms = float(want[want != 0].square().mean().sqrt())
    assert float(off.norm() / want.norm()) <= 3 * spread + storage
    assert float((off - storage * want - 8 * spread * (want + rms)).max()) <= 0, (float(off.max()) / rms, spread)


def check_one_word(torch, O, X, known):
    """The spreads of O and X, {index: (O's, X's)}"""
    spreads = {}
    for i, (a, blocks) in known.items():
        want, s = iterate(a, blocks)
        spread = tolerance(s, max(a.shape), False)[1]
        # of a step's O three steps may share a Gram matrix: twice as much, as in test_gpu_muon.py
        spreads[i] = spread, 2 * spread
        want = torch.from_numpy(want).to("cuda:0")
        close(O[i], want, spread, HALF["f32"])
        close(X[i], want, 2 * spread, HALF["bf16"])
    return spreads


@pytest.mark.parametrize("pair", ONE_WORD_PAIRS, ids=lambda p: name_of(p[0]))
def test_one_word(pair):
    import torch
    groups, others = pair
    O, X, known = orthogonalised(torch, groups, "bf16", "fast", 1)
    spreads = check_one_word(torch, O, X, known)
    P, Y, known_others = orthogonalised(torch, others, "bf16", "fast", 1)
    first = lambda sets: np.cumsum([0] + [count for count, _, _ in sets[:-1]])
    for (_, m, n), i, j in zip(groups, first(groups), first(others)):
        assert np.array_equal(known[i][0], known_others[j][0])
        if 4 * max(m, n) < 5 * min(m, n):                     # step by step
            assert torch.equal(O[i], P[j]) and torch.equal(X[i], Y[j])
        else:
            close(O[i], P[j].double(), math.sqrt(2) * spreads[i][0], 2 * HALF["f32"])
            close(X[i], Y[j].double(), math.sqrt(2) * spreads[i][1], 2 * HALF["bf16"])


@pytest.mark.parametrize("groups", ONE_WORD_SINGLES, ids=name_of)
def test_one_word_on_small_tiles(groups):
    import torch
    check_one_word(torch, *orthogonalised(torch, groups, "bf16", "fast", 3))


@pytest.mark.parametrize("groups", TWO_WORDS, ids=name_of)
def test_two_words(groups):
    import torch
    O, X, known = orthogonalised(torch, groups, "f32", "exact", 2)
    for i, (a, blocks) in known.items():
        want, s = iterate(a, blocks)
        tol = tolerance(s, max(a.shape), True)[0] + HALF["f32"]
        check(O[i], want, tol)
        check(X[i], want, 2 * tol)
        assert not bool(O[i].cpu().numpy()[want == 0].any()) and not bool(X[i].cpu().numpy()[want == 0].any())
