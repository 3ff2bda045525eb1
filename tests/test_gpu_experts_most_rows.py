"""The order of as many choices as rows may be numbered, 2^31 - 2: the last rows' numbers end where 32 bits do."""
import pytest
import torch

import paper_2106_08846_gb300 as bsr

pytestmark = pytest.mark.gpu
N, k = 2 ** 30 - 1, 2


def counts_up(t, first, step=1 << 27):
    """Whether t is first, first + 1, ... (in pieces)."""
    return all(torch.equal(t[i:i + step], torch.arange(first + i, first + min(t.numel(), i + step), dtype=torch.int32, device="cuda"))
               for i in range(0, t.numel(), step))


@pytest.mark.parametrize("align", [1, 3, 1023])
def test_one_expert(align):
    if align == 1:
        n = N
    else:   # the most tokens whose rows, padded to align, are below 2^31
        n = ((2 ** 31 - 1) // align * align - (0 if align == 3 else align - 1)) // k
    x = torch.zeros(n, k, dtype=torch.int32, device="cuda")
    order = bsr.bsr_expert_order(x, 1, align)
    used = -(-n * k // align) * align
    assert order.rows == used < 2 ** 31 and order.offsets.tolist() == [0, used]
    assert counts_up(order.place.view(-1), 0) and counts_up(order.source[:n * k], 0)
    assert (order.source[n * k:] == -1).all()


def test_the_last_expert_of_two():
    """Two experts, every third choice the second's, the last rows behind it without a token."""
    align = 1000
    n = ((2 ** 31 - 1) // align * align - 2 * (align - 1)) // k
    x = torch.zeros(n * k, dtype=torch.int32, device="cuda")
    x[2::3] = 1
    order = bsr.bsr_expert_order(x.view(n, k), 2, align)
    second = x[2::3].numel()
    first = n * k - second
    o1 = -(-first // align) * align
    o2 = o1 + -(-second // align) * align
    assert order.offsets.tolist() == [0, o1, o2] and o2 <= order.rows < 2 ** 31
    place, source = order.place.view(-1), order.source
    assert counts_up(place[2::3], o1) and torch.equal(place[0::3], 2 * torch.arange(place[0::3].numel(), dtype=torch.int32, device="cuda"))
    assert (source[first:o1] == -1).all() and (source[o1 + second:] == -1).all()
    assert torch.equal(source[o1:o1 + second], torch.arange(2, n * k, 3, dtype=torch.int32, device="cuda"))
