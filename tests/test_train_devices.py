"""CPU: every operand of the embedding, the losses and the AdamW step has to live on the current device.  The tensors here only say that
they are on a device, and the library is a stand-in that counts its calls: nothing is launched."""
import pytest
import torch

from paper_2511_00874_b200 import binding as B


class On(torch.Tensor):
    """A tensor that claims to live on the CUDA device ``dev``."""
    dev = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.dev


def on(dev, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(On)
    t.dev = dev
    return t


class Lib:
    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def f(*args):
            if not name.endswith("_bytes"):
                self.calls += 1
            return 256 if name.endswith("_bytes") else 0
        return f


@pytest.fixture
def stub(monkeypatch):
    L = Lib()
    monkeypatch.setattr(B, "lib", lambda: L)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    return L


I, S = torch.int64, torch.int32
LOGITS = dict(logits=((4, 16),), targets=((4,), I), device_status=((1,), S))
VECTORS = lambda *names: {n: ((4,),) for n in names}  # noqa: E731
OPERATORS = {
    "srq_embedding_fwd": dict(table=((9, 16),), ids=((4,), I), out=((4, 16),), device_status=((1,), S)),
    "srq_embedding_bwd": dict(dout=((4, 16),), ids=((4,), I), dtable=((9, 16),), ws=((256,), torch.uint8), device_status=((1,), S)),
    "srq_logprob_fwd": dict(**LOGITS, **VECTORS("logp", "lse")),
    "srq_logprob_bwd": dict(**LOGITS, **VECTORS("lse", "dlogp"), dlogits=((4, 16),)),
    "srq_policy_loss": dict(**LOGITS, **VECTORS("logp_old", "advantage", "weight", "logp_ref", "row_loss", "logp"), loss=((1,),), dlogits=((4, 16),)),
    "srq_preference_loss": dict(**LOGITS, **VECTORS("logp_ref", "logp"), offsets=((3,), I), pair_loss=((1,),), loss=((1,),), dlogits=((4, 16),),
                                ws=((256,), torch.uint8)),
}


@pytest.mark.parametrize("name", OPERATORS)
def test_operands_on_another_device_are_refused(stub, name):
    spec = OPERATORS[name]
    make = lambda where: {n: on(1 if n == where else 0, *s[0], dtype=s[1] if len(s) > 1 else torch.float32) for n, s in spec.items()}  # noqa: E731
    getattr(B, name)(**make(None))
    assert stub.calls == 1
    for operand in spec:
        with pytest.raises(ValueError, match="device"):
            getattr(B, name)(**make(operand))
    assert stub.calls == 1


def entry(n, dev=0, where=None):
    d = lambda name: 1 if name == where else dev  # noqa: E731
    nb = -(-n // 128)
    return B.AdamTensor(on(d("param"), n), on(d("grad"), n), on(d("m"), n, dtype=torch.uint8), on(d("v"), n, dtype=torch.uint8), on(d("m_step"), nb), on(d("v_step"), nb))


def test_tensors_of_a_list_share_a_device(stub):
    for k in (0, 1):
        for where in ("param", "grad", "m", "v", "m_step", "v_step"):
            with pytest.raises(ValueError, match="device"):
                B.AdamTensors([entry(200, where=where if k == 0 else None), entry(40, where=where if k == 1 else None)])
    tensors = B.AdamTensors([entry(200), entry(40)])
    with pytest.raises(ValueError, match="device"):
        tensors.set_grad(1, on(1, 40))
    B.srq_adamw_step(tensors, 1e-3)
    assert stub.calls == 1
    scalars = dict(lr_device=((1,), torch.float32), step_device=((1,), I), grad_scale=((1,), torch.float32), device_status=((1,), S))
    for name, (shape, dtype) in scalars.items():
        with pytest.raises(ValueError, match="device"):
            B.srq_adamw_step(tensors, 1e-3, **{name: on(1, *shape, dtype=dtype)})
    with pytest.raises(ValueError, match="device"):
        B.srq_adamw_step(B.AdamTensors([entry(200, dev=1), entry(40, dev=1)]), 1e-3)
    assert stub.calls == 1


def test_the_step_of_a_quantization_point_is_on_the_current_device(stub):
    B.block_sr(1, 2, step=on(0, 1, dtype=I)).c()
    with pytest.raises(ValueError, match="device"):
        B.block_sr(1, 2, step=on(1, 1, dtype=I)).c()


def test_scalars_without_an_element_are_refused(stub):
    # (their pointer is null, which would mean that the argument was not given)
    tensors = B.AdamTensors([entry(200)])
    for name, dtype, error in (("lr_device", torch.float32, ValueError), ("step_device", I, ValueError), ("grad_scale", torch.float32, ValueError), ("device_status", S, TypeError)):
        with pytest.raises(error):
            B.srq_adamw_step(tensors, 1e-3, **{name: on(0, 0, dtype=dtype)})
    assert stub.calls == 0


def test_a_missing_operand_of_a_list_is_named(stub):
    for name in ("grad", "m", "v", "m_step", "v_step"):
        bad = entry(40)
        setattr(bad, name, None)
        with pytest.raises(ValueError, match=f"tensor 1: {name}"):
            B.AdamTensors([entry(200), bad])
    assert len(B.AdamTensors([])) == 0 and stub.calls == 0


def test_a_weight_that_is_listed_twice_is_refused(stub):
    # two entries would update the same memory at the same time (tied weights are listed once, with the sum of their gradients)
    a, b = entry(200), entry(200)
    for name in ("param", "m", "v", "m_step", "v_step"):
        c = entry(200)
        setattr(c, name, getattr(a, name))
        with pytest.raises(ValueError, match="twice"):
            B.AdamTensors([a, b, c])
    c = entry(200)
    c.grad = a.grad                                                         # read only
    assert len(B.AdamTensors([a, b, c, entry(0), entry(0)])) == 5
