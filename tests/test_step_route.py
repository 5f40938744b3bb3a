"""Routing of many tokens: every share of tokens between workgroups with every number of
experts a lane, groups on whole lanes and across them, biases, both score functions, masked
scores, ties and padding.  Experts and weights of tokens at the borders of what waves, sets
and workgroups take, the order of all choices."""
import numpy as np
import pytest
import torch

import step_plain as plain
from paper_2607_24981_amd import ilw

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]
NONE = plain.NONE


def same(got, want, what):
    got = got.cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape and got.dtype == want.dtype, (what, got.shape, want.shape)
    bad = np.argwhere(got != want)
    assert not bad.size, (what, len(bad), bad[:4], got[got != want][:4], want[got != want][:4])


def at_borders(g, T):
    """The first and last tokens, some on both sides of every kind of border (4, 16, 32, 64
    and runs of 64 tokens up to 256), some anywhere."""
    edges = np.concatenate([np.arange(s, T, s)[[0, -1]] for s in (4, 16, 32, 64, 128, 192, 256, 1024)
                            if s < T])
    edges = np.concatenate([edges, 64 * g.integers(1, max(2, T // 64), 24)])
    t = np.concatenate([[0, 1, 2, T - 2, T - 1], edges - 1, edges, g.integers(0, T, 60)])
    return np.unique(t[(t >= 0) & (t < T)])


# (groups, top_groups) by experts: of whole lanes (span > 0), or not
GROUPS = {200: (8, 3), 256: (8, 4), 300: (4, 2), 512: (16, 5), 1000: (40, 7), 1024: (32, 9)}


WIDTHS = [(63, 7), (96, 6), (200, 5), (256, 8), (300, 32), (512, 10), (1000, 4), (1024, 13)]


CALLS = ([(T, *w) for T in (1025, 4096, 4097, 8193, 16385) for w in WIDTHS]
         # one each of 1, 2, 4, 8 and 16 experts a lane
         + [(50000, *w) for w in WIDTHS if w[0] in (63, 96, 256, 300, 1024)])


@pytest.mark.parametrize("T,E,top_k", CALLS)
def test_many_tokens(T, E, top_k):
    print(f"[gpu] route {T} tokens, {top_k} of {E}", flush=True)
    g = np.random.Generator(np.random.PCG64([T, E]))
    x = np.rint(g.standard_normal((T, E), np.float32) * 130).astype(np.int16)
    x[g.random(T) < 0.03] = NONE                      # padding
    x[T // 2:T // 2 + 70] = NONE                      # a set without any choice
    x[:: 5] = x[:: 5] // 64 * 64                      # ties
    x[:: 7, g.integers(0, E, E // 3)] = NONE          # masked experts
    x[3:: 900, top_k // 2:] = NONE                    # fewer than top_k
    d = ilw.to_device(x)
    bias = g.integers(-(1 << 28), 1 << 28, E).astype(np.int32)
    bias[::9] = 2 ** 31 - 1
    groups, top_groups = GROUPS.get(E, (3, 2))
    few = at_borders(g, T)
    calls = [dict(),  # softmax over all
             dict(bias=bias, sigmoid=True, groups=groups, top_groups=top_groups, group_best=2),
             dict(sigmoid=True, groups=groups, top_groups=top_groups, group_best=1, renormalize=False)]
    # (a call's weights are checked at the borders, its order as a whole)
    for i, kw in enumerate(calls if T < 16385 else calls[:2]):
        b = kw.pop("bias", None)
        r = ilw.ilw_route(d, top_k, bias=None if b is None else ilw.to_device(b), **kw)
        torch.cuda.synchronize()
        want = plain.route(x[few], top_k, b, kw.get("sigmoid", False), kw.get("renormalize", True),
                           kw.get("groups", 1), kw.get("top_groups", 1), kw.get("group_best", 2),
                           1 << 30, 44)
        at = torch.from_numpy(few).cuda()
        same(r.expert[at], want[0], f"call {i}: expert")
        same(r.weight[at], want[1], f"call {i}: weight")
        flat = r.expert.cpu().numpy().reshape(-1)
        assert flat.min() >= -1 and flat.max() < E
        order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
        n = int((flat >= 0).sum())
        rows, slot = np.full(flat.size, -1, np.int32), np.full(flat.size, -1, np.int32)
        rows[:n], slot[order[:n]] = order[:n] // top_k, np.arange(n)
        offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))])
        same(r.offsets, offsets.astype(np.int32), f"call {i}: offsets")
        same(r.rows, rows, f"call {i}: rows")
        same(r.slot, slot.reshape(T, top_k), f"call {i}: slot")


@pytest.mark.parametrize("T,E", [(1500, 256), (9000, 200), (20000, 512)])
def test_weights_of_many_tokens(T, E):
    """Every weight: a token's does not depend on the others, so it is what calls of 500
    tokens give, four tokens a workgroup."""
    print(f"[gpu] route weights {T} tokens, {E} experts", flush=True)
    g = np.random.Generator(np.random.PCG64([9, T, E]))
    x = np.rint(g.standard_normal((T, E), np.float32) * 130).astype(np.int16)
    x[g.random((T, E)) < 0.1] = NONE
    d = ilw.to_device(x)
    bias = ilw.to_device(g.integers(-(1 << 28), 1 << 28, E).astype(np.int32))
    kw = dict(bias=bias, sigmoid=True, groups=8, top_groups=4)
    many = ilw.ilw_route(d, 8, **kw)
    few = [ilw.ilw_route(d[t:t + 500], 8, **kw) for t in range(0, T, 500)]
    torch.cuda.synchronize()
    same(many.expert, torch.cat([r.expert for r in few]).cpu().numpy(), "expert")
    same(many.weight, torch.cat([r.weight for r in few]).cpu().numpy(), "weight")
