"""Entry points of positions, cache pages, masks and differences without a context or descriptors: refused on the host, no GPU needed."""
import ctypes as C
import inspect
import math

import pytest
import torch

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


class _Tensor:
    """What the binding asks of a tensor before it hands its address on."""

    def __init__(self, shape, device=0, contiguous=True, dtype=torch.uint64):
        self.shape, self.device, self.contiguous, self.dtype, self.is_cuda = shape, device, contiguous, dtype, device >= 0

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.device

    def numel(self):
        return math.prod(self.shape)

    def data_ptr(self):
        return 4096


def _context():
    ctx = binding.Context.__new__(binding.Context)
    ctx.log_n, ctx.N, ctx.n, ctx.L, ctx.K, ctx.dnum, ctx.device = 10, 1024, 512, 5, 2, 3, torch.device("cuda", 0)
    return ctx


def test_keys_of_another_shape_or_device_are_refused():
    """A key is read up to its last digit and limb: a shorter one, or one of another context, would be read past its end."""
    ctx, full = _context(), (3, 2, 7, 1024)
    assert ctx._evk(binding.SwitchKey(_Tensor(full), 25), 25).galois == 25
    for bad in ((2, 2, 7, 1024), (3, 2, 6, 1024), (3, 2, 7, 512), (4, 2, 7, 1024), (0,)):
        with pytest.raises(ValueError):
            ctx._evks([binding.SwitchKey(_Tensor(full), 5), binding.SwitchKey(_Tensor(bad), 25)])
    with pytest.raises(ValueError):
        ctx._evks([binding.SwitchKey(_Tensor(full, device=1), 5)])
    for kw in (dict(device=-1), dict(contiguous=False), dict(dtype=torch.int64)):
        with pytest.raises(TypeError):
            ctx._evks([binding.SwitchKey(_Tensor(full, **kw), 5)])


def test_workspaces_of_another_device_are_refused():
    ctx = _context()
    ws = _Tensor((512,), dtype=torch.uint8)
    assert ctx._given(ws) is ws
    for kw in (dict(device=1), dict(device=-1), dict(contiguous=False)):
        with pytest.raises(ValueError):
            ctx._given(_Tensor((512,), dtype=torch.uint8, **kw))


def test_every_call_of_positions_and_maps_checks_its_keys_and_workspace():
    """The methods that hand keys and workspaces on do so through the checks above."""
    for name in ("attention_mask", "attention_difference", "softmax_rows_masked", "_attend", "rotary", "cache_append"):
        source = inspect.getsource(getattr(binding.Context, name))
        assert ("ws: torch.Tensor" not in source and name != "_attend") or "if ws is None else self._given(ws)" in source, name
        assert "rlk.data" not in source and ("keys" not in source or "self._evks(keys)" in source), name
