"""Adjustment of logits after texts of more than 65535 tokens, whose counts pass 16 bits, against double precision with the bounds of
test_gpu_logits_adjust.py (a count is a whole number and exact; frequency times count is one rounding of its magnitude)."""
import pytest
import torch

from test_gpu_logits_adjust import DEV, _case, _check, _check_grad, _gen, _rand, _run

pytestmark = pytest.mark.gpu


def _long_case(n, rows, vocab, typ, lengths, seed=5, distinct=4000):
    """Row texts of these lengths in turn: one token for a third of the places, up to `distinct` others, neighbours among them, and strays."""
    a = _case(n, rows, vocab, typ, seed)
    length = torch.tensor([lengths[r % len(lengths)] for r in range(n * rows)], device=DEV)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), length.cumsum(0)])
    total = int(start[-1])
    text = torch.randint(0, min(vocab, distinct), (total,), device=DEV, generator=_gen(seed + 9)) * max(1, vocab // (2 * distinct))
    text[::3] = vocab - 1
    text[1::50] = torch.tensor([-1, vocab, 2 ** 33, 0], device=DEV).repeat(total)[:text[1::50].numel()]
    a.update(history=text, history_start=start)
    return a


LENGTHS = (70_000, 65_535, 10, 65_536, 0, 200_001)


# short rows; two warps a row; a tile of 16 KB (few long texts among many rows) and of 32 KB, several of them to a row
@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("n,rows,vocab,lengths", [(2, 3, 130, LENGTHS), (1, 6, 777, LENGTHS), (2, 3, 1500, LENGTHS), (1, 3, 5001, LENGTHS),
                                                  (3, 2, 20_000, LENGTHS), (1, 1, 131_072, (100_000,)), (2, 1, 50_001, (65_536, 66_000)),
                                                  (2, 40, 9001, (90_000,) + (3,) * 79)])
def test_many_tokens_many_times(n, rows, vocab, lengths, typ):
    z, d = _rand((n, rows, vocab), 3.0, vocab, typ), _rand((n, rows, vocab), 1.0, vocab + 1, typ)
    a = _long_case(n, rows, vocab, typ, lengths)
    _check(z, typ, a)
    _check_grad(d, z, typ, a)
    for left_out in (("frequency",), ("bias",), ("frequency", "bias", "allowed"), ("presence", "repetition", "bias")):
        _check(z, typ, {k: v for k, v in a.items() if k not in left_out})


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_in_place_wherever_rows_begin(shift, typ):
    vocab = 5001
    z = _rand((1, 4, vocab + 11), 3.0, 1, typ)
    view = z[..., shift:shift + vocab]
    a = _long_case(1, 4, vocab, typ, (70_000, 5, 66_000, 131_072))
    want, around = _run(view.contiguous(), **a), z.clone()
    _run(view, view, **a)
    assert torch.equal(view, want)
    assert torch.equal(z[..., :shift], around[..., :shift]) and torch.equal(z[..., shift + vocab:], around[..., shift + vocab:])
