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
