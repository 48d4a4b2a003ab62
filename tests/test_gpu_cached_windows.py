"""The operators of attention over cached windows together, as a streaming decoder runs them: a window's rows are projected,
its keys and values appended, its queries attend to what is cached."""
import math

import pytest
import torch

from block_ops_util import half_step
from cache_ops_util import attend64, head64, sees
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


class Stream:
    """A cache of one layer for several sequences, and the lists of a call."""

    def __init__(self, seqs, hk, d, page, pages):
        self.kc, self.vc = (torch.full((pages, page, hk, d), math.nan, dtype=BF, device=DEV) for _ in range(2))
        self.table = torch.randperm(pages, device=DEV).to(torch.int32)[: seqs * (pages // seqs)].view(seqs, -1)
        self.lengths = [0] * seqs
        self.page = page

    def step(self, rows, new, hq, pos, widths, gains, **how):
        self.lengths = [a + b for a, b in zip(self.lengths, new)]
        starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=DEV)
        lengths = torch.tensor(self.lengths, dtype=torch.int32, device=DEV)
        hk = self.kc.shape[2]
        q = B.regenvc_paged_append(rows[:, hq:hq + hk], rows[:, hq + hk:], self.kc, self.vc, self.table, lengths, starts,
                                   q=rows[:, :hq], positions=pos, widths=widths, norm=B.NORM_RMS, q_weight=gains[0], k_weight=gains[1])
        return B.regenvc_paged_attn_forward(q, self.kc, self.vc, self.table, lengths, starts, **how)[0]


def test_frames_of_two_streams_then_single_tokens():
    """Windows come in steps of one latent frame, of different sizes for the two streams, then token by token; every step's
    output is that of attention over everything so far, causal by frames, in 64 bits on the values as they were rounded."""
    hq, hk, d, page, widths, frame = 6, 2, 128, 48, [44, 42, 42], 60
    g = torch.Generator().manual_seed(0)
    gains = [(1 + 0.2 * torch.randn(d, generator=g)).to(DEV) for _ in range(2)]
    stream = Stream(2, hk, d, page, 40)
    q_all, k_all, v_all = [[], []], [[], []], [[], []]
    for new in ([60, 60], [60, 0], [60, 120], [1, 1], [1, 0], [0, 1], [58, 7]):
        n = sum(new)
        rows = torch.randn(n, hq + 2 * hk, d, generator=g).to(BF).to(DEV)
        pos = torch.randint(0, 64, (3, n), generator=g, dtype=torch.int32).to(DEV)
        out = stream.step(rows, new, hq, pos, widths, gains, group=frame)
        assert B.regenvc_device_status() == B.OK
        at = 0
        for s, m in enumerate(new):
            part = slice(at, at + m)
            at += m
            if not m:
                continue
            x = rows[part].double()
            turned = [head64(x[:, a:b], w.double(), pos[:, part], widths, 1e4, False, False, 1e-6)[0]
                      for a, b, w in ((0, hq, gains[0]), (hq, hq + hk, gains[1]))]
            q, k = (t.to(BF).double() for t in turned)
            k_all[s].append(k)
            v_all[s].append(x[:, hq + hk:])
            keys = torch.cat(k_all[s])
            ref, _, bound, _ = attend64(q, keys, torch.cat(v_all[s]), sees(m, keys.shape[0], frame, 0), 1 / math.sqrt(d), BF)
            # q and k may round to the neighbouring value here and there: a score is off by at most two half steps of its terms
            slack = 4 * half_step(BF) * (q.abs().amax() * keys.abs().amax() * math.sqrt(d)) * torch.cat(v_all[s]).abs().amax()
            err = (out[part].double() - ref).abs()
            assert (err <= bound + slack).all()
            assert (err <= bound).float().mean() > 0.98


def test_a_whole_window_as_the_windows_own_attention_has_it():
    """Positions of a T x H x W grid and no norm: regenvc_attn_forward's result within both calls' tolerance."""
    T, H, W, h = 3, 10, 16, 4
    n = T * H * W
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, h, 128, generator=g).to(BF).to(DEV) for _ in range(3))
    want = B.regenvc_attn_forward(q, k, v, torch.empty_like(q), T, H, W)
    i = torch.arange(n, device=DEV)
    pos = torch.stack([i // (H * W), i // W % H, i % W]).to(torch.int32)
    stream = Stream(1, h, 128, 64, 10)
    lists = (stream.table, torch.tensor([n], dtype=torch.int32, device=DEV), torch.tensor([0, n], dtype=torch.int32, device=DEV))
    qr = B.regenvc_paged_append(k, v, stream.kc, stream.vc, *lists, q=q, positions=pos, widths=[44, 42, 42])
    got, _ = B.regenvc_paged_attn_forward(qr, stream.kc, stream.vc, *lists)
    assert B.regenvc_device_status() == B.OK
    diff = (got.double() - want.double()).abs()
    assert diff.max() <= 1e-2 * v.double().abs().max()                  # the window's attention is held to that
    assert diff.sum() / want.double().abs().sum() <= 2e-3 + 2 * half_step(BF)   # ... to that, this one rounds q, k and P to bf16


def test_a_captured_step_of_single_tokens():
    """One graph, replayed token by token: the lists, positions and rows change in place."""
    hq, hk, d, page = 4, 2, 64, 16
    g = torch.Generator().manual_seed(2)
    kc, vc = (torch.full((20, page, hk, d), math.nan, dtype=BF, device=DEV) for _ in range(2))
    table = torch.randperm(20, generator=g).to(torch.int32)[:18].view(2, 9).to(DEV)
    rows, pos = torch.zeros(2, hq + 2 * hk, d, dtype=BF, device=DEV), torch.zeros(1, 2, dtype=torch.int32, device=DEV)
    lengths, starts = torch.zeros(2, dtype=torch.int32, device=DEV), torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)

    def step(kc, vc):
        q = B.regenvc_paged_append(rows[:, hq:hq + hk], rows[:, hq + hk:], kc, vc, table, lengths, starts, q=rows[:, :hq],
                                   positions=pos, widths=[d], norm=B.NORM_RMS, halves=True)
        return B.regenvc_paged_attn_forward(q, kc, vc, table, lengths, starts, group=1)[0]

    lengths += 1
    step(kc.clone(), vc.clone())
    lengths -= 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(kc, vc)
    kc.fill_(math.nan), vc.fill_(math.nan)
    kept_k, kept_v = kc.clone(), vc.clone()
    for t in range(40):
        rows.copy_(torch.randn(rows.shape, generator=g))
        pos.fill_(t)
        lengths += 1
        graph.replay()
        want = step(kept_k, kept_v)
        assert torch.equal(out, want) and torch.equal(torch.nan_to_num(kc), torch.nan_to_num(kept_k))
    assert B.regenvc_device_status() == B.OK
