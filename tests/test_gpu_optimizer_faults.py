"""Muon and AdamW on the GPU where a call or its values lie at the edge of what is accepted."""
import math

import numpy as np
import pytest

from oracle.optimizers_oracle import adamw_step, newton_schulz
from paper_2605_16341_amd import binding
from test_gpu_muon import HALF, QUINTIC, check, matrix, tolerance
from test_gpu_muon_tiles import tolerance as tolerances

pytestmark = pytest.mark.gpu


def test_adamw_refuses_a_buffer_given_twice_and_leaves_the_state():
    import torch
    opt = binding.AdamW([64, 0, 64], x_dtype="f32", lr=0.1)
    empty = torch.zeros(0, device="cuda:0")
    a, b, c, d, e, f, g, h = (torch.full((64,), float(k), device="cuda:0") for k in range(1, 9))
    counter = torch.zeros(2, dtype=torch.int32, device="cuda:0")
    call = lambda x, y, m, v: opt.step([x[0], empty, x[1]], [y[0], empty, y[1]], [m[0], empty, m[1]], [v[0], empty, v[1]], counter)
    for lists in (((a, a), (b, c), (d, e), (f, g)), ((a, b), (c, d), (e, e), (f, g)), ((a, b), (c, d), (e, f), (g, g)),
                  ((a, b), (c, d), (e, f), (e, f)), ((a, b), (c, d), (a, e), (f, g)), ((a, b), (c, a), (d, e), (f, g)),
                  ((a, b), (c, d), (d, e), (f, g)), ((a, b), (c, d), (e, f), (g, c))):
        with pytest.raises(ValueError):
            call(*lists)
    assert counter.tolist() == [0, 0] and all(bool((t == k).all()) for k, t in enumerate((a, b, c, d, e, f, g, h), 1))
    call((a, b), (c, c), (d, e), (f, g))
    assert counter.tolist() == [1, 0]


def adamw_once(g, eps, lr=0.25, beta1=0.9, beta2=0.95, t0=0, x0=0.0, m0=0.0, v0=0.0):
    """x, m, v after a step of fp32 tensors in fp64, and what the oracle says of them; the scalars are those that fp32 holds."""
    import torch
    f = lambda a: torch.as_tensor(a, dtype=torch.float32, device="cuda:0").expand(len(g)).contiguous()
    opt = binding.AdamW([len(g)], x_dtype="f32", lr=lr, betas=(beta1, beta2), eps=eps)
    x, grad, m, v = f(x0), f(g), f(m0), f(v0)
    before = [a.double().cpu().numpy() for a in (x, grad, m, v)]
    opt.step([x], [grad], [m], [v], torch.tensor([t0, 0], dtype=torch.int32, device="cuda:0"))
    return [a.double().cpu().numpy() for a in (x, m, v)], adamw_step(*before, t0 + 1, lr, beta1, beta2, float(np.float32(eps)), 0.0)


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1e-30, 1e-8])
def test_adamw_of_tiny_gradients(eps):
    """Second moments below the smallest normal number are held in steps of 2^-149: half a step and the gradient's 2^-24 off, and
    with eps = 0 the step is their root's."""
    g = [s * a for a in (1e-16, 1e-18, 1e-19, 3e-20, 1e-20) for s in (1.0, -1.0)]
    (x, m, v), (wx, wm, wv) = adamw_once(g, eps)
    assert np.all(np.abs(v - wv) <= 2.0 ** -149 + 6 * 2.0 ** -24 * wv)
    # v off by a share e leaves its root e / 2 off; v is corrected in fp32 too, a multiple of 2^-149 again
    share = 2 * (2.0 ** -149 / wv) + 16 * 2.0 ** -24
    assert np.all(np.abs(x - wx) <= share * np.abs(wx)), (x, wx)


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-8])
def test_adamw_without_gradients_stays_with_any_eps(eps):
    (x, m, v), _ = adamw_once([0.0] * 9, eps, x0=0.5)
    assert np.all(x == 0.5) and np.all(m == 0) and np.all(v == 0)


@pytest.mark.parametrize("beta2", [0.95, 0.999])
@pytest.mark.parametrize("t0", [0, 5])
def test_adamw_of_huge_gradients(beta2, t0):
    """Second moments within fp32 whose gradient's square or bias-corrected value lies beyond it."""
    g = [s * a for a in (1e15, 2e19, 5e19) for s in (1.0, -1.0)]
    (x, m, v), (wx, wm, wv) = adamw_once(g, 1e-8, beta2=beta2, t0=t0)
    assert wv.max() < 3e38 < 2.5e39 <= max(g) ** 2
    # four roundings a moment, and of x those of the root, its factor, the sum, the quotient and the products: 16 halves of a step
    assert np.all(np.abs(v - wv) <= 6 * 2.0 ** -24 * wv) and np.all(np.abs(m - wm) <= 4 * 2.0 ** -24 * np.abs(wm))
    assert np.all(np.abs(x - wx) <= 16 * 2.0 ** -24 * np.abs(wx)), (x, wx)


@pytest.mark.parametrize("shape", [(700, 3000), (3000, 700), (1000, 1000), (200, 16384)])
def test_step_of_fp32_parameters_in_fast_precision_is_planned_as_the_orthogonalisation(shape):
    """Fewer Gram matrices than O's own precision admits are for parameters of 8 bits: fp32 ones take the same O, bit by bit, as
    the orthogonalisation gives (both in one word: p^2 q above 2^29)."""
    import torch
    a = torch.randn(*shape, generator=torch.Generator().manual_seed(shape[0])).to("cuda:0", torch.bfloat16)
    opt = binding.Muon([shape], x_dtype="f32", g_dtype="bf16", precision="fast", mu=0.0, lr=-1.0, scale="none")
    o, x, m = (torch.zeros(*shape, device="cuda:0") for _ in range(3))
    opt.orthogonalise([a], [o])
    opt.step([x], [a], [m])
    assert torch.equal(x, o) and bool((o != 0).any())


@pytest.mark.parametrize("shape", [(40, 56), (300, 200), (136, 4096), (600, 1000)])
@pytest.mark.parametrize("coeffs", [((0.02, 0.0, 0.0),) * 5, ((1e-6, 0.0, 0.0),) * 2, ((0.05, -0.03, 0.0), (0.001, 0.0, 0.0), (3.0, 0.0, 0.0), (5.0, 0.0, 0.0)),
                                    ((1e-5, 0.0, 0.0), (12.0, 0.0, 0.0), (12.0, 0.0, 0.0), (12.0, 0.0, 0.0)),
                                    ((7e-8, 0.0, 0.0), (200.0, -100.0, 50.0), (250.0, 0.0, 0.0)), ((30.0, 0.0, 0.0), (7e-8, 0.0, 0.0), (200.0, 0.0, 0.0))])
@pytest.mark.parametrize("precision", ["exact", "fast"])
def test_coefficients_that_shrink(shape, coeffs, precision):
    """Iterates far below 1 keep the bits of their words."""
    import torch
    a = matrix(np.random.default_rng(12), *shape)
    opt = binding.Muon([shape], x_dtype="f32", precision=precision, coeffs=coeffs, mu=0.0, lr=-1.0, scale="none")
    A = torch.from_numpy(a).to("cuda:0", torch.float32)
    o, x, m = (torch.zeros(*shape, device="cuda:0") for _ in range(3))
    opt.orthogonalise([A], [o])
    opt.step([x], [A], [m])
    host = A.double().cpu().numpy()
    want = newton_schulz(host, coeffs)
    for got in (o, x):
        check(got, want, tolerance(host, coeffs, precision == "exact", "f32"))


@pytest.mark.parametrize("coeffs", [((0.0, 0.0, 0.0),), ((0.0, 0.0, 0.0),) + binding.MUON_COEFFS, binding.MUON_COEFFS + ((0.0, 0.0, 0.0),)])
@pytest.mark.parametrize("shape", [(40, 56), (300, 200), (600, 1000)])
def test_a_polynomial_that_is_zero_gives_zeros(coeffs, shape):
    import torch
    opt = binding.Muon([shape], x_dtype="bf16", coeffs=coeffs)
    a = torch.from_numpy(matrix(np.random.default_rng(13), *shape)).to("cuda:0", torch.bfloat16)
    o = torch.ones_like(a)
    opt.orthogonalise([a], [o])
    assert bool((o == 0).all()) and opt.info() == [0]


def test_thin_matrices_beyond_what_steps_together():
    """Rows so long that their padding fills a cluster's workspace with 84 of them: the later ones take it over from the earlier."""
    import torch
    n, count = 400000, 170
    gen = torch.Generator(device="cuda:0").manual_seed(11)
    a = torch.randn(count, 1, n, device="cuda:0", generator=gen).bfloat16()
    o = torch.empty_like(a)
    opt = binding.Muon([(1, n)] * count, x_dtype="bf16")
    assert opt.workspace_bytes < 9 * 10 ** 9
    opt.orthogonalise(list(a), list(o))
    alone = binding.Muon([(1, n)], x_dtype="bf16")
    for k in (0, 1, 82, 83, 84, 85, 167, 168, 169):
        single = torch.empty_like(a[k])
        alone.orthogonalise([a[k]], [single])
        assert torch.equal(o[k], single), k
    assert opt.info() == [0] * count
    # a single row keeps its direction: O is the iteration of 1 times the row over its norm
    s = 1.0
    for ca, cb, cc in binding.MUON_COEFFS:
        s = ca * s + cb * s ** 3 + cc * s ** 5
    want = s * a.double() / a.double().norm(dim=2, keepdim=True)
    # one word of Y and P: 2^-11 twice a step of five; later steps' slopes at s = 0.70, 1.11, 0.72, 1.09 multiply that by 1.42 at most; bf16
    assert float(((o.double() - want).norm(dim=2) / want.norm(dim=2)).max()) <= 10 * 2.0 ** -11 * 2 + 2.0 ** -8


@pytest.mark.parametrize("spectrum", ["1/i", "1/i^2", "rank 1", "rank 8"])
@pytest.mark.parametrize("shape", [(96, 160), (300, 200), (136, 4096), (136, 16384), (520, 1300), (3000, 700), (1000, 1000)])
@pytest.mark.parametrize("g", ["bf16", "f32"])
def test_falling_spectra(spectrum, shape, g):
    """Rounding to u of the largest singular value is u i^2 of the i-th of 1 / i^2, and makes small ones of zeros; the iteration brings all
    of them towards 1: one word leaves 2 % of O on 1 / i^2, 10 % of a matrix of rank 1.  The tolerance is that from the spectrum, by
    the squares of the expected errors."""
    import torch
    rng = np.random.default_rng(31)
    p = min(shape)
    u, v = (np.linalg.qr(rng.standard_normal((d, p)))[0] for d in shape)
    i = np.arange(1.0, p + 1)
    values = {"1/i": 1 / i, "1/i^2": 1 / i ** 2, "rank 1": i <= 1, "rank 8": i <= 8}[spectrum]
    dt = torch.bfloat16 if g == "bf16" else torch.float32
    A = torch.from_numpy((u * values) @ v.T).to("cuda:0", dt)
    host = A.double().cpu().numpy()
    want = newton_schulz(host, QUINTIC)
    s = np.linalg.svd(host / (np.linalg.norm(host) + 1e-7), compute_uv=False)
    spread = tolerances(s, max(shape), g == "f32")[1]
    opt = binding.Muon([shape], x_dtype="f32", g_dtype=g, precision="fast" if g == "bf16" else "exact")
    o = torch.zeros(shape, device="cuda:0")
    opt.orthogonalise([A], [o])
    step = binding.Muon([shape], x_dtype=g, mu=0.0, lr=-1.0, scale="none")
    x, m = torch.zeros_like(A), torch.zeros(shape, device="cuda:0")
    step.step([x], [A], [m])
    for got, room in ((o, 3 * spread + HALF["f32"]), (x, 2 * 3 * spread + HALF[g])):
        off = np.linalg.norm(got.double().cpu().numpy() - want) / np.linalg.norm(want)
        assert off <= room, (off, room)
