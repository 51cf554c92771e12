"""GPU: the stochastic rounding of bfloat16 weights, bit for bit, on weights whose new value is known exactly: without a gradient the step
only shrinks them, p <- round(p (1 - lr weight_decay)), one product in binary32."""
import numpy as np
import pytest
import torch

import _train as ref
import paper_2511_00874_b200 as srq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_weights_are_cut_after_their_threshold(bits):
    n = 1 << 20
    rng = np.random.default_rng(0)
    # every bfloat16 pattern of either sign with each sixteenth of its occurrences another threshold; no NaN, no infinity
    p = torch.from_numpy(((np.arange(n) * 40503) & 0xFFFF).astype(np.uint16).view(np.int16)).view(torch.bfloat16)
    p = torch.where(p.float().isfinite(), p, torch.tensor(1.0, dtype=torch.bfloat16)).cuda()
    decay = np.float32(0.7 + 0.3 * rng.random())
    lr, wd = 2.0 ** -3, float(np.float32((1 - float(decay)) * 8))            # their product is exact
    factor = np.float32(1 - lr * wd)
    x = (p.float().cpu().numpy() * factor).astype(np.float32)
    want = ref.cut_bf16(x, ref.words(n, 7, 3 + (5 << 32)).astype(np.int64) & 0xFFFF)
    t = srq.AdamTensor(p, torch.zeros(n, device="cuda"), *srq.new_adam_state(p, bits))
    s = torch.zeros(1, dtype=torch.int32, device="cuda")
    srq.srq_adamw_step(srq.AdamTensors([t]), lr, weight_decay=wd, step=5, seed=7, tensor_id=3, device_status=s)
    got = t.param.float().cpu().numpy()
    assert s.item() == 0
    bad = got.view(np.uint32) != want.view(np.uint32)
    assert not bad.any(), f"{bad.sum()} off, first: {x[bad][0]!r} became {got[bad][0]!r}, not {want[bad][0]!r}"
