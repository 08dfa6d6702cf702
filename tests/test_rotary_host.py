"""ta_rotary without a GPU: refusals come before any CUDA call, and the reference of the GPU tests has its own pins."""
import ctypes

import numpy as np
import pytest

import paper_2410_20926_b200 as ta
from paper_2410_20926_b200 import api
from rotary_reference import angles, coordinates, rotate


def call(q=1 << 20, k=2 << 20, q_out=3 << 20, k_out=4 << 20, B=1, H=4, H_kv=2, N=8, D=64, sections=(8, 8), **kw):
    if "dims" not in kw and "positions" not in kw:
        kw["positions"] = 5 << 20
    return ta.ta_rotary(q, k, q_out, k_out, B, H, H_kv, N, D, list(sections), stream=0, check=False, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(q=0), "INVALID_ARG"), (dict(q_out=0), "INVALID_ARG"), (dict(k=0), "INVALID_ARG"), (dict(k_out=0), "INVALID_ARG"),
    (dict(H_kv=0), "INVALID_ARG"), (dict(B=0), "INVALID_ARG"), (dict(N=0), "INVALID_ARG"), (dict(H=0), "INVALID_ARG"),
    (dict(D=0), "INVALID_ARG"), (dict(parts=0), "INVALID_ARG"), (dict(sections=(8, -1)), "INVALID_ARG"),
    (dict(sections=[1] * 9), "INVALID_ARG"), (dict(sections=(0, 0)), "SHAPE"), (dict(sections=(16, 17)), "SHAPE"),
    (dict(parts=2, sections=(8, 9)), "SHAPE"), (dict(parts=3), "SHAPE"), (dict(D=512), "UNSUPPORTED"),
    (dict(dtype=2), "UNSUPPORTED"), (dict(base=0.0), "INVALID_ARG"), (dict(base=-1.0), "INVALID_ARG"),
    (dict(base=float("nan")), "INVALID_ARG"), (dict(base=float("inf")), "INVALID_ARG"),
    (dict(positions=None), "INVALID_ARG"), (dict(positions=16, dims=[2, 4]), "INVALID_ARG"),
    (dict(dims=[2, 3]), "SHAPE"), (dict(dims=[2, 4], token_offset=1), "SHAPE"), (dict(dims=[2, 0]), "INVALID_ARG"),
    (dict(dims=[2, 4], token_offset=-1), "INVALID_ARG"), (dict(q=(1 << 20) + 1), "ALIGNMENT"),
    (dict(q_out_strides=(4 * 8 * 64, 0, 64)), "INVALID_ARG"),              # heads of an output share their rows
    (dict(q_out_strides=(4 * 8 * 64, 8 * 64, 63)), "INVALID_ARG"),         # so do its tokens
    (dict(q_out=(1 << 20) + 64), "INVALID_ARG"),                           # an output across its input
    (dict(q_out=2 << 20), "INVALID_ARG"), (dict(k_out=3 << 20), "INVALID_ARG"),
])
def test_refusals(kw, status):
    assert call(**kw) == getattr(ta, "TA_ERR_" + status)


def test_struct_size_is_checked():
    p = api.ta_rotary_params()
    p.struct_bytes = 8
    assert api.load().ta_rotary(ctypes.byref(p)) == ta.TA_ERR_INVALID_ARG
    assert api.load().ta_rotary(None) == ta.TA_ERR_INVALID_ARG


def test_torch_binding_refuses():
    import torch
    q = torch.zeros(1, 2, 4, 16)
    with pytest.raises(ValueError, match="CUDA"):
        ta.multi_axis_rotary(q, q, [4, 4], dims=[2, 2])


def test_reference_is_a_rotation_of_relative_positions():
    """Scores of rotated vectors depend on coordinate differences alone, and the inverse undoes the rotation."""
    rng = np.random.default_rng(3)
    sections, D = (3, 5), 16
    q, k = rng.standard_normal((2, 1, 1, 1, D))
    pos = rng.integers(-50, 50, size=(2, 1, 1))

    def at(x, p, il):
        return rotate(x, angles(p, sections, 100.0, False), 1, il)[0, 0, 0]

    for il in (False, True):
        one = at(q, pos, il) @ at(k, pos + np.array([3, -7]).reshape(2, 1, 1), il)
        two = at(q, pos + 11, il) @ at(k, pos + np.array([14, 4]).reshape(2, 1, 1), il)
        assert abs(one - two) < 1e-12
        ang = angles(pos, sections, 100.0, True)
        assert np.abs(rotate(rotate(q, ang, 1, il), ang, 1, il, inverse=True) - q).max() < 1e-15 * 10
    assert coordinates((2, 3), 4, 1).tolist() == [[0, 0, 1, 1], [1, 2, 0, 1]]
