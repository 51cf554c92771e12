"""GPU: the list of an AdamW step keeps the memory it points to."""
import pytest
import torch

import paper_2511_00874_b200 as srq

pytestmark = pytest.mark.gpu
N = 1 << 20


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("field", ["param", "grad", "m", "v", "m_step", "v_step"])
def test_memory_of_a_listed_tensor_outlives_a_replaced_storage(field, bits):
    if bits == 32 and field.endswith("_step"):
        pytest.skip("32-bit moments have no step sizes")
    p = torch.randn(N, device="cuda")
    t = srq.AdamTensor(p, torch.randn(N, device="cuda"), *srq.new_adam_state(p, bits))
    a = srq.AdamTensors([t])
    old = getattr(t, field)
    kept, new = old.clone(), old.clone()
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    old.data = new
    assert torch.cuda.memory_allocated() == held                            # else the step below would go to memory that is no longer its own
    # and goes where the list says
    srq.srq_adamw_step(a, 1e-3, step=1)
    assert torch.equal(new, kept)


def test_a_gradient_that_is_given_anew_frees_the_old_one():
    p = torch.randn(N, device="cuda")
    a = srq.AdamTensors([srq.AdamTensor(p, torch.randn(N, device="cuda"), *srq.new_adam_state(p))])
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for _ in range(3):
        a.set_grad(0, torch.randn(N, device="cuda"))
    assert torch.cuda.memory_allocated() == held
    del a
    assert torch.cuda.memory_allocated() < held
