"""The operators behind a decoder step's attention as they are used: one after another
as a layer of experts and a vocabulary head, in captured graphs, on several streams and
with workspaces of any content; what the binding refuses."""
import numpy as np
import pytest
import torch

import decoder_plain
import step_plain as plain
from paper_2607_24981_amd import ilw

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]
NONE = plain.NONE


def say(msg):
    print(f"[gpu] {msg}", flush=True)


def dev(a):
    return ilw.to_device(a)


def same(got, want, what):
    got = got.cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape and got.dtype == want.dtype, (what, got.shape, want.shape)
    assert np.array_equal(got, want), (what, np.count_nonzero(got != want), got.size)


def rng(*seed):
    return np.random.Generator(np.random.PCG64(seed))


# tokens [T, D] -> experts (hidden H) -> tokens -> log probabilities of V
SHAPES = [dict(T=1, D=64, E=8, top=2, H=96, V=112), dict(T=70, D=128, E=16, top=3, H=64, V=48),
          dict(T=150, D=48, E=5, top=5, H=80, V=64)]


def layer(g, D, E, top, H, V, T):
    """Weights and factors of a layer."""
    def scaled(*shape, out):
        k = shape[-1]
        shift = 30 + int(round(np.log2(42 * 73 * np.sqrt(k) / out)))
        return (g.integers(-127, 128, shape).astype(np.int8),
                g.integers(1 << 29, 1 << 30, shape[:-1]).astype(np.int32),
                np.full(shape[:-1], shift, np.int32))
    w = {"router": scaled(-(-E // 16) * 16, D, out=130),  # whole 16s; the rest is cut off
         "up": scaled(E, H, D, out=40),
         "down": scaled(E, D, H, out=600), "head": scaled(V, D, out=190)}
    k = H
    w["static"] = (g.integers(-127, 128, (E, D, k)).astype(np.int8),
                   g.integers(1 << 29, 1 << 30, (E, D)).astype(np.int32),
                   np.full((E, D), 30 + int(round(np.log2(42 * 73 * np.sqrt(k) / 40))), np.int32))
    return w


def tokens(g, T, D):
    return np.rint(g.normal(0, 1, (T, D)) * np.exp2(g.uniform(4, 10, (T, 1)))).astype(np.int16)


def run_plain(w, x, pad, given, top):
    T, D = x.shape
    q, s = plain.quantize_rows(x)

    def linear(q, s, name, bits, offsets=None, rows=None, M=None):
        W, mult, shift = w[name]
        W, mult, shift = (W, mult, shift) if offsets is not None else (W[None], mult[None], shift[None])
        M = q.shape[0] if M is None else M
        y = np.zeros((M, W.shape[1]), np.int16 if bits == 16 else np.int8)
        plain.linear_scaled(q, s, W, None, mult, shift, [0, M] if offsets is None else offsets.tolist(),
                            rows, bits, y)
        return y
    scores = linear(q, s, "router", 16)[:, :w["up"][0].shape[0]]
    scores[pad] = NONE
    r = plain.route(scores, top, None, True, True, 1, 1, 2, 1 << 30, 44)
    expert, weight, offsets, rows, slot = r
    h = linear(q, s, "up", 16, offsets, rows, rows.size)
    hq, hs = plain.quantize_rows(h)
    d = linear(hq, hs, "down", 16, offsets, None, rows.size)
    y = plain.combine(d, slot, weight, 1 << 22, 30, x, 1 << 30)
    yq, ys = plain.quantize_rows(y)
    lp = plain.log_probs(linear(yq, ys, "head", 16), given, 5)
    # the same experts with factors fixed beforehand, int8 throughout
    h8 = linear(q, s, "up", 8, offsets, rows, rows.size)
    W, mult, shift = w["static"]
    d8 = np.zeros((rows.size, D), np.int8)
    decoder_plain.grouped(h8, None, offsets.tolist(), W, None, mult, shift, d8)
    y8 = plain.combine(d8, slot, weight, 1 << 22, 30, None, 0)
    return (*r, y, *lp, y8)


class Layer:
    """The same on the device; rows that no token has are cleared first."""

    def __init__(self, w, top):
        self.w = {k: [dev(v) for v in t] for k, t in w.items()}
        self.top = top

    def linear(self, q, s, name, **kw):
        W, mult, shift = self.w[name]
        return ilw.ilw_linear_scaled(q, s, W, None, mult, shift, **kw)

    def __call__(self, x, pad, given):
        q, s = ilw.ilw_quantize_rows(x)
        scores = self.linear(q, s, "router")[:, :self.w["up"][0].shape[0]]
        scores.masked_fill_(pad.unsqueeze(1), NONE)
        r = ilw.ilw_route(scores, self.top, sigmoid=True)
        M, D = r.rows.numel(), x.shape[1]

        def rows_of(n, dtype):
            return torch.zeros(M, n, dtype=dtype, device="cuda")
        H = self.w["up"][0].shape[1]
        h = self.linear(q, s, "up", offsets=r.offsets, rows=r.rows, y=rows_of(H, torch.int16))
        hq, hs = ilw.ilw_quantize_rows(h)
        d = self.linear(hq, hs, "down", offsets=r.offsets, y=rows_of(D, torch.int16))
        y = ilw.ilw_combine(d, r.slot, r.weight, 1 << 22, 30, skip=x, skip_mult=1 << 30)
        yq, ys = ilw.ilw_quantize_rows(y)
        lp = ilw.ilw_log_probs(self.linear(yq, ys, "head"), given, top=5)
        h8 = self.linear(q, s, "up", offsets=r.offsets, rows=r.rows, bits=8, y=rows_of(H, torch.int8))
        W, mult, shift = self.w["static"]
        d8 = ilw.ilw_linear_grouped(h8, W, r.offsets, None, mult, shift, y=rows_of(D, torch.int8))
        y8 = ilw.ilw_combine(d8, r.slot, r.weight, 1 << 22, 30)
        return (*r, y, *lp, y8)


NAMES = ("expert", "weight", "offsets", "rows", "slot", "y", "given", "entropy", "top",
         "top_log_prob", "y8")


def inputs(g, T, D, V):
    pad = g.random(T) < 0.1
    return tokens(g, T, D), pad, g.integers(0, V, (T, 2)).astype(np.int32)


def check(got, want, what):
    for name, a, b in zip(NAMES, got, want):
        same(a, b, f"{what}: {name}")


@pytest.mark.parametrize("shape", SHAPES)
def test_layer(shape):
    g = rng(shape["T"])
    w = layer(g, **shape)
    x, pad, given = inputs(g, shape["T"], shape["D"], shape["V"])
    say(f"layer {shape}")
    got = Layer(w, shape["top"])(dev(x), dev(pad), dev(given))
    torch.cuda.synchronize()
    check(got, run_plain(w, x, pad, given, shape["top"]), str(shape))


def test_layer_captured_and_replayed():
    """A graph replayed over new inputs, eager work and synchronizations between."""
    shape = SHAPES[1]
    g = rng(21)
    w = layer(g, **shape)
    net = Layer(w, shape["top"])
    sets = [inputs(g, shape["T"], shape["D"], shape["V"]) for _ in range(4)]
    want = [run_plain(w, *s, shape["top"]) for s in sets]
    held = [dev(v) for v in sets[0]]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        net(*held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = net(*held)
    say("layer replayed")
    for i in (0, 1, 2, 3, 1):
        for h, v in zip(held, sets[i]):
            h.copy_(dev(v))
        for o in out:
            o.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        check(out, want[i], f"replay {i}")
        check(net(*[dev(v) for v in sets[(i + 1) % 4]]), want[(i + 1) % 4], f"eager after {i}")


def test_layers_on_two_streams():
    """Two layers at a time, each with its own workspaces."""
    parts = []
    for i, shape in enumerate(SHAPES[1:]):
        g = rng(31, i)
        w = layer(g, **shape)
        x = inputs(g, shape["T"], shape["D"], shape["V"])
        parts.append((Layer(w, shape["top"]), [dev(v) for v in x],
                      run_plain(w, *x, shape["top"]), torch.cuda.Stream()))
    torch.cuda.synchronize()
    say("two streams")
    got = []
    for _ in range(6):
        for net, x, _, stream in parts:
            with torch.cuda.stream(stream):
                got.append(net(*x))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        check(out, parts[i % 2][2], f"call {i}")


@pytest.mark.parametrize("fill", [0, -1, 0x5A])
def test_workspaces_hold_anything(fill):
    """Exactly the size asked for, any content."""
    g = rng(41)
    x = np.rint(g.normal(0, 130, (500, 24))).astype(np.int16)
    need = ilw.lib().ilw_route_workspace_bytes(500, 24)
    ws = torch.full((need,), fill, dtype=torch.int8, device="cuda")
    say(f"workspaces {fill}")
    r = ilw.ilw_route(dev(x), 4, workspace=ws)
    for name, a, b in zip(r._fields, r, plain.route(x, 4, None, False, True, 1, 1, 2, 1 << 30, 44)):
        same(a, b, name)
    s = np.rint(g.normal(0, 192, (3, 120000))).astype(np.int16)
    given = g.integers(0, 120000, (3, 2)).astype(np.int32)
    need = ilw.lib().ilw_log_probs_workspace_bytes(3, 120000, 9)
    assert need > 0
    ws = torch.full((need,), fill, dtype=torch.int8, device="cuda")
    lp = ilw.ilw_log_probs(dev(s), dev(given), top=9, workspace=ws)
    for name, a, b in zip(lp._fields, lp, plain.log_probs(s, given, 9)):
        same(a, b, name)
    with pytest.raises(ilw.IlwError, match="status -5"):
        ilw.ilw_log_probs(dev(s), dev(given), top=9, workspace=ws[:-16])


def test_stage_timing():
    g = rng(51)
    shape = SHAPES[0]
    w = layer(g, **shape)
    x = [dev(v) for v in inputs(g, shape["T"], shape["D"], shape["V"])]
    net = Layer(w, shape["top"])
    net(*x)
    ilw.profile_enable(True)
    try:
        net(*x)
        got = ilw.profile_read()
    finally:
        ilw.profile_enable(False)
    count = {k: n for k, (ms, n) in got.items() if n}
    assert count == {"quantize": 3, "gemm_scaled": 5, "route": 1, "combine": 2, "log_probs": 1,
                     "gemm_grouped": 1}
    assert all(got[k][0] > 0 for k in count)


def test_binding_refuses():
    def z(*shape, dtype=torch.int8):
        return torch.zeros(*shape, dtype=dtype, device="cuda")
    i16, i32 = torch.int16, torch.int32
    x16, x8, w = z(4, 64, dtype=i16), z(4, 64), z(32, 64)
    s, m = z(4, dtype=i32), torch.ones(32, dtype=i32, device="cuda")
    slot = z(4, 2, dtype=i32)
    bad = [
        lambda: ilw.ilw_quantize_rows(x8), lambda: ilw.ilw_quantize_rows(x16.cpu()),
        lambda: ilw.ilw_quantize_rows(x16.t()), lambda: ilw.ilw_quantize_rows(x16[0]),
        lambda: ilw.ilw_quantize_rows(x16[:, :40]), lambda: ilw.ilw_quantize_rows(x16[:, 1:49]),
        lambda: ilw.ilw_quantize_rows(x16, y=z(4, 32)),
        lambda: ilw.ilw_quantize_rows(x16[:1].expand(4, 64)),
        lambda: ilw.ilw_linear_scaled(x16, s, w, None, m, m),
        lambda: ilw.ilw_linear_scaled(x8, s[:3], w, None, m, m),
        lambda: ilw.ilw_linear_scaled(x8, s, w.view(1, 32, 64), None, m, m),
        lambda: ilw.ilw_linear_scaled(x8, s, w, None, m, m, offsets=s),
        lambda: ilw.ilw_linear_scaled(x8, s, w.view(2, 16, 64), None, m, m, offsets=s),
        lambda: ilw.ilw_linear_scaled(x8, s, w, m[:5], m, m),
        lambda: ilw.ilw_linear_scaled(x8, s, w, None, m, m[:5]),
        lambda: ilw.ilw_linear_scaled(x8, s, w, None, m[:5], m[:5]),
        lambda: ilw.ilw_linear_scaled(x8, s, w, None, m, m, bits=32),
        lambda: ilw.ilw_linear_scaled(x8, s, w, None, m, m, y=z(4, 32)),
        lambda: ilw.ilw_linear_scaled(x8, s, z(32, 48), None, m, m),
        lambda: ilw.ilw_route(x8, 2), lambda: ilw.ilw_route(x16, 0), lambda: ilw.ilw_route(x16, -1),
        lambda: ilw.ilw_route(x16, 33), lambda: ilw.ilw_route(x16, 2, bias=s),
        lambda: ilw.ilw_route(x16, 2, groups=3), lambda: ilw.ilw_route(x16.t(), 2),
        lambda: ilw.ilw_route(x16[:1].expand(4, 64), 2),
        lambda: ilw.ilw_combine(x8, slot, s, 1, 1), lambda: ilw.ilw_combine(s, slot, slot, 1, 1),
        lambda: ilw.ilw_combine(x8, slot, slot, 1, 0),
        lambda: ilw.ilw_combine(x8, slot, slot, 1, 1, skip=x16),
        lambda: ilw.ilw_combine(x8, slot, slot, 1, 1, skip=z(3, 64)),
        lambda: ilw.ilw_combine(x8, slot, slot.to(torch.int64), 1, 1),
        lambda: ilw.ilw_log_probs(x8), lambda: ilw.ilw_log_probs(x16, top=65),
        lambda: ilw.ilw_log_probs(x16, top=-1), lambda: ilw.ilw_log_probs(x16, given=s),
        lambda: ilw.ilw_log_probs(x16, top=-1, workspace=x8.view(-1)),
        lambda: ilw.ilw_log_probs(x16, given=slot[:3]),
        lambda: ilw.ilw_log_probs(x16, given=slot.to(torch.int64)),
        lambda: ilw.ilw_log_probs(x16, given=z(4, 65, dtype=i32)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(ilw.IlwError):
            f()
            print("not refused:", i)
    torch.cuda.synchronize()


def test_empty_calls():
    """No rows, no tokens, nothing asked for."""
    def z(*shape, dtype=torch.int8):
        return torch.zeros(*shape, dtype=dtype, device="cuda")
    i16, i32 = torch.int16, torch.int32
    y, s = ilw.ilw_quantize_rows(z(0, 64, dtype=i16))
    assert y.shape == (0, 64) and s.shape == (0,)
    m = torch.ones(32, dtype=i32, device="cuda")
    assert ilw.ilw_linear_scaled(y, s, z(32, 64), None, m, m).shape == (0, 32)
    assert ilw.ilw_combine(z(0, 64), z(0, 2, dtype=i32), z(0, 2, dtype=i32), 1, 1).shape == (0, 64)
    r = ilw.ilw_log_probs(z(0, 64, dtype=i16), z(0, 3, dtype=i32), top=4)
    assert r.given.shape == (0, 3) and r.top.shape == (0, 4)
    r = ilw.ilw_log_probs(z(3, 64, dtype=i16))
    assert r.given.shape == (3, 0) and r.entropy.tolist() == [6 << 16] * 3 and r.top.shape == (3, 0)
    torch.cuda.synchronize()
