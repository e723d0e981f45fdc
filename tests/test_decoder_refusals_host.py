"""Further refusals of the operators between the layers: caches that differ in type, numbers that fp32 does not hold (no GPU needed)."""
import ctypes

import pytest

from paper_2602_06694_amd import binding as nq

A = 1 << 20            # an address that is never followed: every call here is refused before anything is launched


def test_caches_of_different_types_are_not_moved_together():
    a, b = (nq.nq_kv_create(A, A, t, 2, 64, 16, 8) for t in (nq.NQ_BF16, nq.NQ_F16))
    both = (ctypes.c_void_p * 2)(a, b)
    assert nq.lib().nq_kv_copy_pages(both, 2, A, A, 0, None) == nq.NQ_E_INVALID_ARG
    assert nq.lib().nq_kv_compact(both, 2, A, A, 4, A, 4, A, 0, None) == nq.NQ_E_INVALID_ARG
    for h in (a, b):
        nq.nq_kv_destroy(h)


@pytest.mark.parametrize("scale,cap", [(1e39, 0.0), (-1e300, 0.0), (3e38, 0.0), (1.0, 1e-50), (1.0, 1e-39), (1.0, 1e39), (1.0, 3e38), (1.0, 1e300), (1e10, 1e-30), (1e-3, 1e38), (1e-60, 1.0)])
def test_scales_and_caps_that_fp32_does_not_hold(scale, cap):
    """A cap that rounds to zero would be none, one beyond fp32 would make NaN of all scores."""
    kv = nq.nq_kv_create(A, A, nq.NQ_BF16, 2, 64, 16, 8)
    with pytest.raises(nq.NQError) as e:
        nq.nq_attn_create(kv, 4, scale, cap, nq.NQ_F32)
    assert e.value.status == nq.NQ_E_INVALID_ARG
    nq.nq_kv_destroy(kv)


@pytest.mark.parametrize("scale,cap", [(1.0, 0.0), (0.0, 0.0), (-0.125, 0.0), (0.0, 30.0), (-0.125, 30.0), (0.125, 1e30), (0.125, 1e-30), (1e-60, 0.0), (2e38, 0.0)])
def test_scales_and_caps_that_are_taken(scale, cap):
    kv = nq.nq_kv_create(A, A, nq.NQ_BF16, 2, 64, 16, 8)
    nq.nq_attn_destroy(nq.nq_attn_create(kv, 4, scale, cap, nq.NQ_F32))
    nq.nq_kv_destroy(kv)


@pytest.mark.parametrize("change", [dict(magnitude=1e39), dict(magnitude=-1e300), dict(eps=1e39), dict(weight_offset=1e60), dict(weight_offset=-4e38)])
def test_rotations_of_numbers_that_fp32_does_not_hold(change):
    """They are held in 32 bits: what is finite in binary64 alone would be an infinity there."""
    a = dict(q_heads=4, kv_heads=2, head_dim=64, rot_dim=0, layout=nq.NQ_ROPE_HALF, inv_freq=None, magnitude=1.0, eps=1e-6, weight_offset=0.0, in_dtype=nq.NQ_F32,
             out_dtype=nq.NQ_BF16)
    with pytest.raises(nq.NQError) as e:
        nq.nq_rope_create(**{**a, **change})
    assert e.value.status == nq.NQ_E_INVALID_ARG
