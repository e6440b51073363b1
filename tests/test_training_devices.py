"""The training operators take tensors of one device: a kernel cannot read another card's memory, and a call that mixed them would end in
a fault.  Stand-ins for tensors, since the machine may have no card or one: a refused call looks at no address."""
import pytest
import torch

from paper_2312_17530_amd import binding as b


class OnCard:
    """What the binding asks of a tensor."""

    def __init__(self, *shape, dtype=torch.float32, device=0):
        self.shape, self.dtype, self.device_index = torch.Size(shape), dtype, device
        self.is_cuda = device >= 0

    def get_device(self):
        return self.device_index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def stride(self):
        out = [1]
        for n in reversed(self.shape[1:]):
            out.insert(0, out[0] * n)
        return tuple(out)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x7000_0000_0000


def _args(name, top=3):
    bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    x, row = lambda: OnCard(4, 16, dtype=bf16), lambda: OnCard(4, dtype=f32)  # noqa: E731
    ws = lambda: OnCard(1 << 24, dtype=torch.uint8)  # noqa: E731
    head = dict(x=x(), w=OnCard(10, 16, dtype=bf16))
    grads = dict(lse=row(), row_grad=row(), dx=x(), dw=OnCard(160, dtype=f32), accumulate=False, workspace=ws())
    taught = dict(top_idx=OnCard(4, top, dtype=i32), top_logit=OnCard(4, top, dtype=f32), temperature=2.0)
    return {"rsdgc_layer_norm": dict(x=x(), gamma=OnCard(16), beta=OnCard(16), eps=1e-5, y=x(), mean=row(), rstd=row()),
            "rsdgc_layer_norm_backward": dict(dy=x(), x=x(), gamma=OnCard(16), mean=row(), rstd=row(), dx=x(), dgamma=OnCard(16), dbeta=OnCard(16),
                                              accumulate=False, workspace=ws()),
            "rsdgc_head_loss": head | dict(target=OnCard(4, dtype=i32), loss=row(), lse=row(), workspace=ws()),
            "rsdgc_head_loss_backward": head | dict(target=OnCard(4, dtype=i32)) | grads,
            "rsdgc_distill_loss": head | taught | dict(loss=row(), lse=row(), workspace=ws()),
            "rsdgc_distill_loss_backward": head | taught | grads}[name]


NAMES = ["rsdgc_layer_norm", "rsdgc_layer_norm_backward", "rsdgc_head_loss", "rsdgc_head_loss_backward", "rsdgc_distill_loss", "rsdgc_distill_loss_backward"]
MIXED = [(name, k, device) for name in NAMES for k, v in _args(name).items() if isinstance(v, OnCard) for device in (1, -1)]


class Reached(Exception):
    pass


@pytest.fixture
def no_call(monkeypatch):
    """The library's calls, replaced: what reaches them is not launched."""
    lib = b._training()
    for name in NAMES:
        def reached(*args):
            raise Reached
        monkeypatch.setattr(lib, name, reached)
    monkeypatch.setattr(b, "_stream_on", lambda t, stream: None)


@pytest.mark.parametrize("name,which,device", MIXED, ids=[f"{n}-{k}-{d}" for n, k, d in MIXED])
def test_a_tensor_of_another_device_is_refused(no_call, name, which, device):
    args = _args(name)
    args[which].device_index, args[which].is_cuda = device, device >= 0
    with pytest.raises(b.RsdgcError):
        getattr(b, name)(**args)


@pytest.mark.parametrize("device", [0, 1])
@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_one_device_reach_the_library(no_call, name, device):
    args = _args(name)
    for v in args.values():
        if isinstance(v, OnCard):
            v.device_index = device
    with pytest.raises(Reached):
        getattr(b, name)(**args)
