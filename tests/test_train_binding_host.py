"""What the binding of the training operators refuses before an address reaches the library, without a GPU."""
import pytest
import torch

from paper_2104_11981_b200 import binding as B


class Tensor:
    """As much of a CUDA tensor as gradients_build looks at; nothing reads its address."""
    is_cuda, dtype = True, torch.float32

    def __init__(self, index, address, count=8):
        self.device, self.address, self.count = torch.device("cuda", index), address, count

    def is_contiguous(self):
        return True

    def numel(self):
        return self.count

    def data_ptr(self):
        return self.address


def test_gradients_are_on_the_current_device(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for host in (torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16)):
        with pytest.raises(AssertionError):
            B.gradients_build([[host]])
        with pytest.raises(AssertionError):
            B.gradients_build([[Tensor(0, 1 << 20)], [host]])
    with pytest.raises(AssertionError):
        B.gradients_build([[Tensor(0, 1 << 20), Tensor(1, 1 << 21)]])
    with pytest.raises(AssertionError):
        B.gradients_build([[Tensor(0, 1 << 20)], [Tensor(1, 1 << 21)]])
    with pytest.raises(AssertionError):
        B.gradients_build([[Tensor(1, 1 << 20)], [Tensor(1, 1 << 21)]])
    if not torch.cuda.is_available():                    # a host-only handle
        assert B.gradients_build([[Tensor(0, 1 << 20)], [Tensor(0, 1 << 21)]]).columns == 8


def test_empty_lists_are_refused():
    for nodes in ([], [[]], [[], []]):
        with pytest.raises(B.DecentlamError) as e:
            B.gradients_build(nodes)
        assert e.value.status == -2
