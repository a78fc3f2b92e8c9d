"""Equal logits in greedy rows: the lowest index, wherever the equal ones lie among the values before the first 16-byte boundary of a piece of
the row, its 16-byte units, and the values behind the last."""
import pytest

from _gpu import ct

pytestmark = pytest.mark.gpu

TYPES = ["float32", "float16", "bfloat16"]


def first_best(x):
    return (x == x.amax(dim=1, keepdim=True)).int().argmax(dim=1)       # argmax of equal integers: the first


def greedy(x, drafts, offsets, most):
    import torch
    batch = offsets.shape[0] - 1
    got = ct().ct_verify_drafts(x, drafts, offsets, most, torch.zeros(drafts.shape[0], device="cuda"), torch.ones(batch, x.shape[1], device="cuda"),
                                temperature=torch.zeros(batch, device="cuda"))
    return got[0].tolist(), got[1].tolist()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 11, 13, 2055, 32003])
@pytest.mark.parametrize("start", [0, 1, 3])
def test_two_equal_values(vocab, dtype, start):
    """Every pair of a short row; in a long one the last values against some of its units."""
    import torch
    lows = range(vocab - 1) if vocab < 20 else [0, 1, 5, 8, 17, vocab // 2, vocab - 20, vocab - 9]
    pairs = [(i, j) for i in lows for j in range(max(i + 1, vocab - 9), vocab)]
    store = torch.zeros(2 * len(pairs), vocab + start, dtype=getattr(torch, dtype), device="cuda")
    x = store[:, start:]
    for r, (i, j) in enumerate(pairs):
        x[2 * r, i] = x[2 * r, j] = 1.0
    offsets = torch.arange(len(pairs) + 1, device="cuda")
    low, high = (torch.tensor([p[k] for p in pairs], device="cuda") for k in (0, 1))
    accepted, token = greedy(x, low, offsets, 1)
    assert accepted == [1] * len(pairs) and [t[0] for t in token] == [p[0] for p in pairs] and all(t[1] == 0 for t in token)
    accepted, token = greedy(x, high, offsets, 1)                       # the higher of the two is not the answer: it falls
    assert accepted == [0] * len(pairs) and [t[0] for t in token] == [p[0] for p in pairs]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 17, 129, 1003, 2051, 9001, 50001])
def test_rows_of_few_values(vocab, dtype):
    """Many equal values in each row."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(vocab)
    for start in (0, 1, 2, 5):
        x = torch.randint(0, 1 + vocab // 3, (40, vocab + start), device="cuda", generator=g).clamp(max=200).to(getattr(torch, dtype))[:, start:]
        offsets = torch.zeros(41, dtype=torch.int64, device="cuda")
        accepted, token = greedy(x, offsets[:0], offsets, 0)
        assert accepted == [0] * 40 and [t[0] for t in token] == first_best(x).tolist()
