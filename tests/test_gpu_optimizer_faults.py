"""Muon and AdamW on the GPU where a call or its values lie at the edge of what is accepted."""
import pytest

from paper_2605_16341_amd import binding

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
