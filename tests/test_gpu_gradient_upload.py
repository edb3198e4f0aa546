"""A gradient list used at once on a stream that nothing orders behind the one that its table was copied on."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tensors", [3, 3000])
def test_first_call_on_an_unordered_stream(tensors):
    """Tables of a few pieces and of 12,000; norms of ones are exact."""
    from paper_2104_11981_b200 import binding as B
    n = 4
    g = torch.ones((n, tensors, 7 if tensors > 3 else 80_000), device="cuda:0")
    norms, side = torch.full((n,), float("nan"), device="cuda:0"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        lst = B.gradients_build([[g[i, t] for t in range(tensors)] for i in range(n)])
        B.gradient_norm(lst, norms, stream=side)
        side.synchronize()
        assert np.array_equal(norms.cpu().numpy(), np.full(n, np.float32(np.sqrt(g[0].numel()))))
        norms.fill_(float("nan"))
        torch.cuda.synchronize()
        lst.destroy()
