"""Calls of about as many items as there are thread blocks, which take them whole or cut them."""
import math

import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def lists(table, lengths, starts):
    return tuple(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lengths, starts))


@pytest.mark.parametrize("heads,rows", [(33, 1024), (36, 1000), (37, 1024), (132, 256), (147, 256), (148, 200), (149, 256),
                                        (71, 300), (18, 2048), (19, 2000), (1, 37888), (1, 37700)])
def test_about_as_many_items_as_thread_blocks(heads, rows):
    """With and without whole items in rounds: rows are alike whichever head they are computed for."""
    g = torch.Generator().manual_seed(heads)
    n, d = rows + 40, 64
    k, v = (torch.randn(n, 1, d, generator=g).to(BF).to(DEV).expand(n, heads, d).contiguous() for _ in range(2))
    q = torch.randn(rows, 1, d, generator=g).to(BF).to(DEV)
    where = lists([list(range(-(-n // 64)))], [n], [0, rows])
    caches = []
    for t in (k, v):
        c = torch.zeros(-(-n // 64) * 64, heads, d, dtype=BF, device=DEV)
        c[:n] = t
        caches.append(c.view(-1, 64, heads, d))
    out, _ = B.regenvc_paged_attn_forward(q.expand(rows, heads, d).contiguous(), *caches, *where, group=1)
    one, _ = B.regenvc_paged_attn_forward(q, *(c[:, :, :1].contiguous() for c in caches), *where, group=1)
    assert B.regenvc_device_status() == B.OK
    s = (q[:, 0].double() @ k[:, 0].double().t()) / math.sqrt(d)
    s = s.masked_fill(torch.arange(n, device=DEV) > torch.arange(n - rows, n, device=DEV)[:, None], -math.inf)
    want = torch.softmax(s, dim=1) @ v[:, 0].double()
    size = torch.softmax(s, dim=1) @ v[:, 0].double().abs()
    bound = (2.0 ** -8 + 2e-4) * size + 2.0 ** -8 * want.abs()   # a rounding of a weight and of the result; fp32 scores and sums
    assert ((out.double() - want[:, None]).abs() <= bound[:, None]).all()
    assert ((one[:, 0].double() - want).abs() <= bound).all()
