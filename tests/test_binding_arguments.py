"""CPU-only checks of the binding's own handling of arguments, before anything reaches the library."""
import ctypes

import pytest

from paper_2605_16341_amd import binding as b

FAKE = 1 << 20            # an aligned "device address", never dereferenced


def status_of(call):
    with pytest.raises(b.OrthDionError) as e:
        call()
    return e.value.status


@pytest.mark.parametrize("ptrs,want", [([], []), ([FAKE], [FAKE]), ([FAKE, 2 ** 64 - 8], [FAKE, 2 ** 64 - 8]), ([None, FAKE], [None, FAKE]),
                                       ([ctypes.c_void_p(FAKE), FAKE], [FAKE, FAKE]), ([-8, 0], [2 ** 64 - 8, None]), ((FAKE, None), [FAKE, None])])
def test_addresses(ptrs, want):
    assert list(b._ptr_array(ptrs)) == want


def test_null_addresses_reach_the_library():
    """None stands for a null pointer: refused by the library where there is something behind it, taken for an empty tensor."""
    h = b.orthdion_create([(64, 64)], 8, b.ORTHDION_F32, b.ORTHDION_F32)
    need = b.orthdion_workspace_bytes(h)
    for k in range(4):
        ptrs = [[None] if i == k else [FAKE] for i in range(4)]
        assert status_of(lambda: b.orthdion_step(h, *ptrs, FAKE, need)) == b.ORTHDION_E_NULL_PTR
    b.orthdion_destroy(h)
    h = b.orthdion_muon_create([(64, 64)], b.ORTHDION_F32, b.ORTHDION_F32)
    assert status_of(lambda: b.orthdion_muon_step(h, [None], [FAKE], [FAKE], FAKE, b.orthdion_muon_workspace_bytes(h))) == b.ORTHDION_E_NULL_PTR
    b.orthdion_muon_destroy(h)
    h = b.orthdion_adamw_create([5, 0], b.ORTHDION_F32, b.ORTHDION_F32)
    some, odd = [FAKE, None], [FAKE + 2, None]
    assert status_of(lambda: b.orthdion_adamw_step(h, [None, None], some, some, some, FAKE)) == b.ORTHDION_E_NULL_PTR
    assert status_of(lambda: b.orthdion_adamw_step(h, some, odd, some, some, FAKE)) == b.ORTHDION_E_MISALIGNED      # not the empty one's null
    b.orthdion_adamw_destroy(h)


@pytest.mark.parametrize("ptrs", [["8"], [1.5], [object()]])
def test_what_is_no_address_is_refused(ptrs):
    with pytest.raises(TypeError):
        b._ptr_array(ptrs)


def test_adamw_refuses_a_buffer_given_twice():
    """Addresses of the four lists of a step over tensors of 4, 6 and 0 elements; the empty one's may be any."""
    opt = b.AdamW([4, 6, 0], x_dtype="f32")
    good = [[64, 128, 0], [192, 256, 0], [320, 384, 0], [448, 512, 0]]          # X, G, M, V
    opt._separate_tensors(*good)
    opt._separate_tensors(good[0], [192, 192, 64], good[2], good[3])           # gradients are only read
    for written in (0, 2, 3):
        twice = [list(seq) for seq in good]
        twice[written][1] = twice[written][0]
        with pytest.raises(ValueError):
            opt._separate_tensors(*twice)
        for other in (0, 1, 2, 3):
            if other != written:
                shared = [list(seq) for seq in good]
                shared[other][0] = shared[written][1]
                with pytest.raises(ValueError):
                    opt._separate_tensors(*shared)


QUINTIC, CUBIC, CONVERGING = ((3.4445, -4.7750, 2.0315),) * 5, ((1.5, -0.5, 0.0),) * 10, ((1.875, -1.25, 0.375),) * 14
STEEP = ((8.28721, -23.59589, 17.30039), (4.10706, -2.94785, 0.54484), (3.94869, -2.90890, 0.55182), (3.31842, -2.48849, 0.51005), (2.30065, -1.66890, 0.41881))


@pytest.mark.parametrize("coeffs,taken", [
    (QUINTIC, True), (CUBIC, True), (CONVERGING, True), (((1.0, 0.0, 0.0),), True), (((0.05, 0.0, 0.0),) * 4, True),
    # the last step's result is fp32 or bf16
    (((0.02, 0.0, 0.0),) * 5, True), (((1e-6, 0.0, 0.0),), True), (((1e-6, 0.0, 0.0),) * 2, True),
    (((0.0, 0.0, 0.0),), True), (((0.0, 0.0, 0.0),) + QUINTIC, True),
    (((0.01, 0.0, 0.0),) * 5, False), (((0.01, 0.0, 0.0),) * 8, False), (((1e-6, 0.0, 0.0),) * 3, False), (((1e-8, 0.0, 0.0),), False),
    # 2 % a step for rounding: singular values just beyond 1 run away from this one
    (STEEP, False), (tuple((x / 1.02, y / 1.02 ** 3, z / 1.02 ** 5) for x, y, z in STEEP), True)])
def test_muon_coefficients(coeffs, taken):
    if taken:
        b.orthdion_muon_destroy(b.orthdion_muon_create([(64, 64)], b.ORTHDION_BF16, b.ORTHDION_BF16, coeffs=coeffs))
    else:
        assert status_of(lambda: b.orthdion_muon_create([(64, 64)], b.ORTHDION_BF16, b.ORTHDION_BF16, coeffs=coeffs)) == b.ORTHDION_E_INVALID_ARG


@pytest.mark.parametrize("coeffs", [((1.0, 0.0), (0.0, 1.0, 0.0, 0.0)), ((1.0, 0.0, 0.0, 0.0), (1.0, 0.0)), ((1.0, 0.0),), ((1.0, 0.0, 0.0),) * 33])
def test_muon_coefficients_are_triples(coeffs):
    with pytest.raises(ValueError):
        b.orthdion_muon_create([(64, 64)], b.ORTHDION_BF16, b.ORTHDION_BF16, coeffs=coeffs)


@pytest.mark.parametrize("shape,count", [((4, 100000), 1000), ((1, 4000000), 100), ((100000, 4), 1000), ((1, 512), 1 << 17), ((129, 129), 32000)])
@pytest.mark.parametrize("dtype", [b.ORTHDION_BF16, b.ORTHDION_F32])
def test_muon_workspace_of_many_thin_matrices_is_bounded(shape, count, dtype):
    """At most 2^29 elements of 8 words of two bytes (two words a value in fp32) step together, or one matrix, beside the tables:
    a matrix's pointers, shape and 256 sums."""
    def need(n):
        h = b.orthdion_muon_create([shape] * n, dtype, dtype)
        got = b.orthdion_muon_workspace_bytes(h)
        b.orthdion_muon_destroy(h)
        return got
    words = 1 if dtype == b.ORTHDION_BF16 else 2
    assert need(count) <= max(2 ** 29 * 8 * 2 * words, need(1)) + count * 2300 + 2048
