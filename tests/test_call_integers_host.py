"""Whole numbers of the training operators' calls beyond 32 bits are refused like any other that is too large, not cut."""
import pytest

from paper_2104_11981_b200 import binding as B

BIG = 1 << 20
CALLERS = sorted({B._calls, B._lib}, key=str)


@pytest.mark.parametrize("calls", CALLERS)
def test_numbers_beyond_32_bits(calls):
    """2^32 + 2 nodes are not two, and 2^32 is not type 0."""
    def norm(n=2, dtype=0, eps=-1.0):
        return calls.layer_norm(n, 3, 8, BIG, dtype, 8, 2 * BIG, 8, None, 0, eps, 3 * BIG, 8, 4 * BIG, 5 * BIG, 0)
    assert norm() == -5
    assert norm(n=(1 << 32) + 2) == -8 and norm(n=(1 << 31) + 1) == -8 and norm(n=-(1 << 32) + 2) == -2 and norm(dtype=1 << 32) == -6

    def grad(n=2, dtype=0, gtype=0):
        return calls.layer_norm_grad(n, 3, 8, BIG, dtype, 8, BIG, 7, BIG, 8, BIG, BIG, BIG, 8, BIG, 8, None, 0, gtype, BIG, BIG, 0)
    assert grad() == -2 and grad(n=(1 << 32) + 2) == -8 and grad(dtype=1 << 32) == -6 and grad(gtype=(1 << 40) + 1) == -6

    def policy(n=2, dtype=0):
        return calls.policy_loss_grad(n, 3, 100, BIG, dtype, 99, BIG, BIG, BIG, BIG, None, 0.2, 0.2, 0.0, BIG, BIG, None, 0, BIG, 256, 0)
    assert policy() == -2 and policy(n=(1 << 32) + 2) == -8 and policy(dtype=1 << 32) == -6


def test_workspaces_of_too_many_nodes():
    for call in (B.layer_norm_grad_workspace_bytes, B.policy_loss_workspace_bytes):
        with pytest.raises(B.DecentlamError) as e:
            call((1 << 32) + 1, 1, 1)
        assert e.value.status == -8
