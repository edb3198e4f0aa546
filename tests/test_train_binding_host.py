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


class OnGpu:
    """A host tensor that says it is on the GPU."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_workspaces_have_the_bytes_that_they_say(monkeypatch):
    """An expanded tensor counts bytes that it does not hold, a strided one lies between those of others."""
    reached = []

    class Calls:
        def __getattr__(self, name):
            return lambda *args: reached.append(name) or 0

    monkeypatch.setattr(B, "_calls", Calls())
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    n, rows, c = 2, 3, 16
    on = lambda *shape, **kw: OnGpu(torch.zeros(shape, **kw))  # noqa: E731
    x, w, stat, need = on(n, rows, c), on(n, c), on(n, rows), B.layer_norm_grad_workspace_bytes(n, rows, c)
    policy = (x, on(n, rows, dtype=torch.int64), stat, stat, stat, None, 0.2, 0.2, 0.0, on(n), stat, x)
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(need), torch.zeros(2 * need, dtype=torch.uint8)[::2]):
        with pytest.raises(AssertionError):
            B.layer_norm_grad(x, x, w, stat, stat, x, w, w, OnGpu(bad))
        with pytest.raises(AssertionError):
            B.policy_loss_grad(*policy, OnGpu(bad))
    assert reached == []
    B.layer_norm_grad(x, x, w, stat, stat, x, w, w, on(need, dtype=torch.uint8))
    B.policy_loss_grad(*policy, on(need, dtype=torch.uint8))
    assert reached == ["layer_norm_grad", "policy_loss_grad"]
