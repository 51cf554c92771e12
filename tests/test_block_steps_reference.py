"""CPU: refusals of a quantization point with a step's number on the device."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2511_00874_b200 import binding

P = 1 << 20                      # an "aligned pointer": the calls below must return before it is used


@pytest.fixture(scope="module")
def L():
    entry.build()
    return binding.lib()


def point(**kw):
    q = binding.block_sr(1, 2).c()
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def test_a_misaligned_step_is_refused(L):
    b = binding._Blocks(P, 256, P, 4, 1)
    ref = ctypes.byref
    for q in (point(step_device=P + 4), point(step_device=P + 1, round=binding.RNE)):
        assert int(L.srq_quantize_blocks(P, 1, 128, 256, 256, ref(q), ref(b), None, None, None)) == binding.ERR_INVALID_ARG
        assert int(L.srq_requantize_blocks(ref(b), 128, 256, ref(q), ref(b), None, None, None)) == binding.ERR_INVALID_ARG
        assert int(L.srq_rmsnorm_fwd(P, 256, None, 0, 1, P, 1, 128, 256, 1e-5, ref(q), ref(b), None, 0, None, 0, None, None, None)) == binding.ERR_INVALID_ARG
        assert int(L.srq_glu_bwd(P, 1, 256, ref(b), ref(b), 128, 256, 0, ref(q), ref(b), None, None, None, None, None, None)) == binding.ERR_INVALID_ARG


def test_other_quantizers_have_no_step(L):
    q = binding.QSpec().c()
    q.step_device = P
    ref = ctypes.byref
    assert int(L.sr_quantize(P, 0, 8, 8, 8, ref(q), P, 8, P, None, 0, None, P, 1 << 20, None)) == binding.ERR_UNSUPPORTED
    assert int(L.sr_quantize_static(P, 0, 8, 8, 8, ref(q), P, 8, P, None, 0, None, None, None)) == binding.ERR_UNSUPPORTED
    good = binding.QSpec().c()
    for a, b in ((q, good), (good, q)):
        assert int(L.qlinear_fwd(P, P, 0, 32, 32, 32, ref(a), ref(b), P, None, P, 1 << 30, None)) == binding.ERR_UNSUPPORTED


def test_a_step_has_to_be_one_whole_number_on_the_device():
    for t in (torch.zeros(1, dtype=torch.int64), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), torch.zeros(0, dtype=torch.int64)):
        with pytest.raises(ValueError, match="step"):
            binding.block_sr(1, 2, step=t).c()
