"""Entry points of positions, cache pages, masks and differences without a context or descriptors: refused on the host, no GPU needed."""
import ctypes as C

import pytest

from paper_2609_12378_b200 import binding


def _null(argtypes):
    return [0 if t in (C.c_uint32, C.c_uint64, C.c_size_t, C.c_int64) else 0.0 if t is C.c_double else None for t in argtypes]


@pytest.mark.parametrize("name", ["ckks_rotary_table", "ckks_rotary_rotations", "ckks_rotary", "ckks_cache_append", "ckks_attention_mask",
                                  "ckks_attention_difference", "ckks_softmax_rows_masked", "ckks_attention_masked", "ckks_attention_differential"])
def test_null_arguments_are_refused(name):
    f = getattr(binding.load(), name)
    assert f(*_null(f.argtypes)) == binding.ERR_ARG


@pytest.mark.parametrize("name", ["ckks_rotary_workspace_bytes", "ckks_cache_append_workspace_bytes", "ckks_attention_mask_workspace_bytes",
                                  "ckks_attention_difference_workspace_bytes", "ckks_attention_masked_workspace_bytes",
                                  "ckks_attention_differential_workspace_bytes"])
def test_no_workspace_without_a_context(name):
    f = getattr(binding.load(), name)
    assert f(*_null(f.argtypes)) == 0


def test_descriptors_have_the_header_s_size():
    assert C.sizeof(binding.CAttnMask) == 24 and C.sizeof(binding.CRotaryDesc) == 24 and C.sizeof(binding.CCacheSpan) == 12
    assert C.sizeof(binding.CRotaryScaling) == 8 + 6 * 8
