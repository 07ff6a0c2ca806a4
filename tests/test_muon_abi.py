"""CPU-only checks of the Muon and AdamW entry points: arguments are validated before the GPU is touched."""
import ctypes
import math

import pytest

from paper_2605_16341_amd import binding as b

FAKE = 1 << 20            # an aligned "device address", never dereferenced


def status_of(call):
    with pytest.raises(b.OrthDionError) as e:
        call()
    return e.value.status


def test_muon_create_takes_any_shape_and_refuses_empty_ones():
    for shape in ((1, 1), (1, 4000), (4000, 1), (17, 33), (64, 64), (8192, 8192)):
        h = b.orthdion_muon_create([shape], b.ORTHDION_BF16, b.ORTHDION_BF16)
        assert b.orthdion_muon_workspace_bytes(h) > 0
        b.orthdion_muon_destroy(h)
    for shape in ((0, 4), (4, 0), (-1, 4), (1 << 22, 4)):
        assert status_of(lambda: b.orthdion_muon_create([shape], 1, 1)) == b.ORTHDION_E_BAD_SHAPE
    for lds in ((15, 16, 16), (16, 15, 16), (16, 16, 15)):
        assert status_of(lambda: b.orthdion_muon_create([(8, 16)], 1, 1, lds=[lds])) == b.ORTHDION_E_BAD_SHAPE
    assert status_of(lambda: b.orthdion_muon_create([], 1, 1)) == b.ORTHDION_E_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(mu=1.5), dict(mu=-0.1), dict(mu=math.nan), dict(lr=math.inf), dict(weight_decay=math.nan),
                                dict(eps=-1e-9), dict(eps=math.inf), dict(precision=5), dict(coeffs=()), dict(scales=[math.nan]),
                                dict(coeffs=((math.nan, 0, 0),)), dict(coeffs=((40.0, 0.0, 0.0),)),
                                dict(coeffs=((8.0, 0.0, 0.0),) * 3), dict(coeffs=((300.0, -400.0, 100.0),))])
def test_muon_create_refuses(kw):
    assert status_of(lambda: b.orthdion_muon_create([(64, 64)], 1, 1, **kw)) == b.ORTHDION_E_INVALID_ARG


def test_muon_create_refuses_types_and_too_many_steps():
    assert status_of(lambda: b.orthdion_muon_create([(64, 64)], 3, 1)) == b.ORTHDION_E_INVALID_ARG
    assert status_of(lambda: b.orthdion_muon_create([(64, 64)], 1, 3)) == b.ORTHDION_E_INVALID_ARG
    with pytest.raises(ValueError):
        b.orthdion_muon_create([(64, 64)], 1, 1, coeffs=((1.0, 0.0, 0.0),) * 33)
    with pytest.raises(ValueError):
        b.orthdion_muon_create([(64, 64)], 1, 1, coeffs=((1.0, 0.0),))


def test_muon_calls_reject_bad_buffers_before_launching():
    h = b.orthdion_muon_create([(64, 48)], b.ORTHDION_BF16, b.ORTHDION_F32)
    need = b.orthdion_muon_workspace_bytes(h)
    step = lambda x=FAKE, g=FAKE, m=FAKE, ws=FAKE, size=need: b.orthdion_muon_step(h, [x], [g], [m], ws, size)
    orth = lambda a=FAKE, o=FAKE, ws=FAKE, size=need: b.orthdion_muon_orthogonalise(h, [a], [o], ws, size)
    for call in (step, orth):
        assert status_of(lambda: call(ws=0)) == b.ORTHDION_E_NULL_PTR
        assert status_of(lambda: call(size=need - 1)) == b.ORTHDION_E_WORKSPACE_TOO_SMALL
        assert status_of(lambda: call(ws=FAKE + 16)) == b.ORTHDION_E_MISALIGNED
    for kw in (dict(x=0), dict(g=0), dict(m=0)):
        assert status_of(lambda: step(**kw)) == b.ORTHDION_E_NULL_PTR
    for kw in (dict(x=FAKE + 1), dict(g=FAKE + 2), dict(m=FAKE + 2)):
        assert status_of(lambda: step(**kw)) == b.ORTHDION_E_MISALIGNED
    for kw in (dict(a=0), dict(o=0)):
        assert status_of(lambda: orth(**kw)) == b.ORTHDION_E_NULL_PTR
    assert status_of(lambda: b.orthdion_muon_get_info(h, 1)) == b.ORTHDION_E_NO_STEP
    for bad in (lambda: b.orthdion_muon_set_lr(h, math.nan), lambda: b.orthdion_muon_set_mu(h, 1.01),
                lambda: b.orthdion_muon_set_weight_decay(h, math.inf)):
        assert status_of(bad) == b.ORTHDION_E_INVALID_ARG
    b.orthdion_muon_set_lr(h, 0.5)
    b.orthdion_muon_set_mu(h, 0.0)
    b.orthdion_muon_set_weight_decay(h, 0.1)
    b.orthdion_muon_destroy(h)


def test_null_handles():
    lib = b.load()
    assert lib.orthdion_muon_create(None, None, 1, None) == b.ORTHDION_E_NULL_PTR
    assert lib.orthdion_adamw_create(None, None, 1, None) == b.ORTHDION_E_NULL_PTR
    h = ctypes.c_void_p()
    assert lib.orthdion_muon_create(ctypes.byref(h), None, 1, None) == b.ORTHDION_E_NULL_PTR
    assert lib.orthdion_adamw_create(ctypes.byref(h), None, 1, None) == b.ORTHDION_E_NULL_PTR
    assert lib.orthdion_muon_workspace_bytes(None) == 0
    assert lib.orthdion_muon_destroy(None) == b.ORTHDION_E_NULL_PTR and lib.orthdion_adamw_destroy(None) == b.ORTHDION_E_NULL_PTR
    assert lib.orthdion_muon_set_lr(None, 0.1) == b.ORTHDION_E_NULL_PTR and lib.orthdion_adamw_set_lr(None, 0.1) == b.ORTHDION_E_NULL_PTR


def test_muon_workspace_is_shared_by_clusters():
    """A set beyond what steps together needs no more than its largest part and the tables."""
    def need(count):
        h = b.orthdion_muon_create([(4096, 4096)] * count, 1, 1)
        got = b.orthdion_muon_workspace_bytes(h)
        b.orthdion_muon_destroy(h)
        return got
    assert need(2) > 1.9 * need(1)
    assert need(64) < need(32) + 64 * 4096


@pytest.mark.parametrize("kw", [dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(lr=math.inf),
                                dict(eps=-1.0), dict(weight_decays=[math.nan]), dict(lr_scales=[math.inf])])
def test_adamw_create_refuses(kw):
    assert status_of(lambda: b.orthdion_adamw_create([16], 1, 1, **kw)) == b.ORTHDION_E_INVALID_ARG


def test_adamw_refusals():
    assert status_of(lambda: b.orthdion_adamw_create([], 1, 1)) == b.ORTHDION_E_INVALID_ARG
    assert status_of(lambda: b.orthdion_adamw_create([-1], 1, 1)) == b.ORTHDION_E_BAD_SHAPE
    assert status_of(lambda: b.orthdion_adamw_create([1 << 42], 1, 1)) == b.ORTHDION_E_BAD_SHAPE
    assert status_of(lambda: b.orthdion_adamw_create([4], 2, 1)) == b.ORTHDION_E_INVALID_ARG
    h = b.orthdion_adamw_create([5, 0], b.ORTHDION_BF16, b.ORTHDION_F32)
    step = lambda x=FAKE, g=FAKE, m=FAKE, v=FAKE, c=FAKE: b.orthdion_adamw_step(h, [x, 0], [g, 0], [m, 0], [v, 0], c)
    for kw in (dict(x=0), dict(g=0), dict(m=0), dict(v=0), dict(c=0)):
        assert status_of(lambda: step(**kw)) == b.ORTHDION_E_NULL_PTR
    for kw in (dict(x=FAKE + 1), dict(g=FAKE + 2), dict(m=FAKE + 1), dict(v=FAKE + 2), dict(c=FAKE + 2)):
        assert status_of(lambda: step(**kw)) == b.ORTHDION_E_MISALIGNED
    assert status_of(lambda: b.orthdion_adamw_set_lr(h, math.nan)) == b.ORTHDION_E_INVALID_ARG
    b.orthdion_adamw_set_lr(h, 0.5)
    b.orthdion_adamw_destroy(h)


def test_classes_refuse_wrong_tensors():
    import torch
    opt = b.AdamW([4, 6], x_dtype="f32", lr=0.1)
    cpu = [torch.zeros(4), torch.zeros(6)]
    with pytest.raises(ValueError):
        opt.step(cpu, cpu, cpu, cpu, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        b.AdamW([4, 6], weight_decay=[0.1])
    with pytest.raises(ValueError):
        b.AdamW([4], x_dtype="f16")
    for kw in (dict(scale="sqrt"), dict(scale=[1.0, 2.0]), dict(lds=[]), dict(x_dtype="f16")):
        with pytest.raises(ValueError):
            b.Muon([(8, 8)], device="cpu", **kw)
    muon = b.Muon([(8, 8)], x_dtype="f32", device="cpu")
    t = [torch.zeros(8, 8)]
    for call in (lambda: muon.step(t, t, t), lambda: muon.step(t, t, []), lambda: muon.orthogonalise(t, t)):
        with pytest.raises(ValueError):
            call()
