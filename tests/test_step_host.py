"""The operators behind a decoder step's attention on the CPU: refusals, found on the
host before anything is launched, workspace sizes, the plain forms themselves, and what
the built kernels keep in memory."""
import ctypes

import numpy as np
import pytest

import step_plain as plain
from paper_2607_24981_amd import ilw
from test_kernel_resources import kernels, named  # noqa: F401

OK, E_NULL, E_SHAPE, E_PARAM, E_UNSUP, E_WS = 0, -1, -2, -3, -4, -5
FAKE = 0x10000  # aligned, never dereferenced: every call below fails or has nothing to do


def check(rc, code):
    assert rc == code, (rc, code, ilw.last_error())
    assert bool(ilw.last_error()) == (code != OK)


@pytest.mark.parametrize("kw,code", [
    (dict(M=0), OK), (dict(M=-1), E_SHAPE), (dict(K=0, ld=0), E_SHAPE), (dict(K=24), E_SHAPE),
    (dict(K=(1 << 20) + 16, ld=1 << 21), E_SHAPE), (dict(ld=56), E_SHAPE), (dict(ld=68), E_SHAPE),
    (dict(x=None), E_NULL), (dict(y=None), E_NULL), (dict(scale=None), E_NULL),
    (dict(x=FAKE + 2), E_PARAM), (dict(y=FAKE + 8), E_PARAM), (dict(M=1 << 30), E_UNSUP),
    (dict(M=1 << 24, K=8192, ld=8192), E_UNSUP)])
def test_quantize_refusals(kw, code):
    f = dict(x=FAKE, ld=64, y=FAKE, scale=FAKE, M=3, K=64)
    f.update(kw)
    check(ilw.lib().ilw_quantize_rows(*f.values(), None), code)


@pytest.mark.parametrize("kw,code", [
    (dict(M=0), OK), (dict(M=-1), E_SHAPE), (dict(x_rows=-1), E_SHAPE), (dict(x_rows=3), E_SHAPE),
    (dict(x_rows=0, rows=FAKE), E_SHAPE), (dict(N=40), E_SHAPE), (dict(K=72), E_SHAPE),
    (dict(N=0), E_SHAPE), (dict(K=131088), E_UNSUP), (dict(experts=0), E_SHAPE),
    (dict(experts=1025), E_SHAPE), (dict(experts=2, offsets=None, n=1), E_SHAPE),
    (dict(y_bits=32), E_PARAM), (dict(y_bits=0), E_PARAM), (dict(x=None), E_NULL),
    (dict(x_scale=None), E_NULL), (dict(w=None), E_NULL), (dict(y=None), E_NULL),
    (dict(mult=None), E_NULL), (dict(shift=None), E_NULL), (dict(n=7), E_SHAPE),
    (dict(n=95, experts=2), E_SHAPE), (dict(x=FAKE + 8), E_PARAM),
    (dict(w=FAKE + 8), E_PARAM), (dict(y=FAKE + 2), E_PARAM),
    (dict(M=1 << 29, x_rows=1 << 30), E_UNSUP), (dict(M=1 << 31, x_rows=1 << 32), E_UNSUP),
    (dict(experts=1024, N=1 << 22), E_UNSUP)])
def test_linear_refusals(kw, code):
    f = dict(x=FAKE, x_rows=4, x_scale=FAKE, rows=None, offsets=FAKE, w=FAKE, b=None, mult=FAKE,
             shift=FAKE, n=48, y=FAKE, y_bits=16, M=4, experts=1, N=48, K=64)
    f.update(kw)
    rq = ilw.Dyadic(f.pop("mult"), f.pop("shift"), f.pop("n"))
    v = list(f.values())
    check(ilw.lib().ilw_linear_scaled(*v[:7], rq, *v[7:], None), code)


ROUTE = dict(top_k=4, groups=1, top_groups=1, group_best=2, sigmoid=0, renormalize=1,
             weight_mult=1 << 30, weight_shift=44)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=-1), E_SHAPE), (dict(experts=0), E_SHAPE), (dict(experts=1025, ld=2000), E_SHAPE),
    (dict(ld=63), E_SHAPE), (dict(rp=False), E_NULL), (dict(top_k=0), E_PARAM),
    (dict(top_k=33), E_PARAM), (dict(top_k=8, experts=7), E_PARAM), (dict(groups=0), E_PARAM),
    (dict(groups=65, experts=65, ld=65), E_PARAM), (dict(groups=3), E_PARAM),
    (dict(top_groups=0), E_PARAM), (dict(groups=4, top_groups=5), E_PARAM),
    (dict(group_best=0), E_PARAM), (dict(group_best=3), E_PARAM), (dict(sigmoid=2), E_PARAM),
    (dict(renormalize=-1), E_PARAM), (dict(weight_mult=-1), E_PARAM),
    (dict(weight_shift=0), E_PARAM), (dict(weight_shift=63), E_PARAM),
    (dict(tokens=1 << 29), E_UNSUP), (dict(offsets=None), E_NULL), (dict(logits=None), E_NULL),
    (dict(expert=None), E_NULL), (dict(weight=None), E_NULL), (dict(rows=None), E_NULL),
    (dict(slot=None), E_NULL), (dict(ws=None), E_WS), (dict(size=-1), E_WS),
    (dict(ws=FAKE + 4), E_PARAM)])
def test_route_refusals(kw, code):
    f = dict(logits=FAKE, ld=64, bias=None, expert=FAKE, weight=FAKE, offsets=FAKE, rows=FAKE,
             slot=FAKE, tokens=200, experts=64)
    rp = ilw.RouteParams(*[kw.get(k, v) for k, v in ROUTE.items()])
    f.update({k: v for k, v in kw.items() if k in f})
    need = ilw.lib().ilw_route_workspace_bytes(200, 64)
    assert need > 0 and ilw.lib().ilw_route_workspace_bytes(32, 64) == 0
    check(ilw.lib().ilw_route(*f.values(), None if kw.get("rp") is False else ctypes.byref(rp),
                              kw.get("ws", FAKE), need + kw.get("size", 0), None), code)


def test_workspace_refusals():
    L = ilw.lib()
    for args in ((-1, 8), (8, 0), (8, 1025)):
        assert L.ilw_route_workspace_bytes(*args) == 0 and ilw.last_error()
    for args in ((-1, 8, 1), (8, 0, 1), (8, (1 << 20) + 1, 1), (8, 8, 65), (8, 8, -1), (1 << 22, 8, 1)):
        assert L.ilw_log_probs_workspace_bytes(*args) == 0 and ilw.last_error()
    assert L.ilw_log_probs_workspace_bytes(0, 1 << 20, 64) == 0 and not ilw.last_error()
    assert L.ilw_log_probs_workspace_bytes(1, 1 << 20, 64) > 0


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=0), OK), (dict(tokens=-1), E_SHAPE), (dict(v_rows=-1), E_SHAPE),
    (dict(N=24), E_SHAPE), (dict(N=0), E_SHAPE), (dict(N=1 << 24), E_SHAPE),
    (dict(top_k=0), E_SHAPE), (dict(top_k=33), E_SHAPE), (dict(bits=4), E_PARAM),
    (dict(mult_a=-2 ** 31), E_PARAM), (dict(mult_b=-2 ** 31), E_PARAM), (dict(shift=0), E_PARAM),
    (dict(shift=63), E_PARAM), (dict(v=None), E_NULL), (dict(slot=None), E_NULL),
    (dict(weight=None), E_NULL), (dict(y=None), E_NULL), (dict(v=FAKE + 8), E_PARAM),
    (dict(skip=FAKE + 8), E_PARAM), (dict(y=FAKE + 4), E_PARAM), (dict(tokens=1 << 31), E_UNSUP),
    (dict(tokens=1 << 62), E_UNSUP)])
def test_combine_refusals(kw, code):
    f = dict(v=FAKE, bits=8, v_rows=4, slot=FAKE, weight=FAKE, skip=FAKE, mult_a=5, mult_b=5,
             shift=20, y=FAKE, tokens=3, top_k=2, N=48)
    f.update(kw)
    check(ilw.lib().ilw_combine(*f.values(), None), code)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=0), OK), (dict(rows=-1), E_SHAPE), (dict(vocab=0), E_SHAPE),
    (dict(vocab=(1 << 20) + 1, ld=1 << 21), E_SHAPE), (dict(n_top=65), E_SHAPE),
    (dict(n_top=-1), E_SHAPE), (dict(n_given=65), E_SHAPE), (dict(n_given=-1), E_SHAPE),
    (dict(ld=299999), E_SHAPE), (dict(logits=None), E_NULL), (dict(entropy=None), E_NULL),
    (dict(given=None), E_NULL), (dict(given_lp=None), E_NULL), (dict(top=None), E_NULL),
    (dict(top_lp=None), E_NULL), (dict(rows=1 << 22), E_UNSUP), (dict(ws=None), E_WS),
    (dict(size=-1), E_WS), (dict(ws=FAKE + 8), E_PARAM)])
def test_log_probs_refusals(kw, code):
    f = dict(logits=FAKE, ld=300000, given=FAKE, n_given=2, given_lp=FAKE, entropy=FAKE, top=FAKE,
             top_lp=FAKE, rows=3, vocab=300000, n_top=5)
    f.update({k: v for k, v in kw.items() if k in f})
    need = ilw.lib().ilw_log_probs_workspace_bytes(3, 300000, 5)
    assert need > 0
    check(ilw.lib().ilw_log_probs(*f.values(), kw.get("ws", FAKE), need + kw.get("size", 0), None),
          code)


# ------------------------------------------------- the plain forms themselves
def test_plain_quantize_is_the_nearest_code():
    g = np.random.Generator(np.random.PCG64(1))
    x = g.integers(-20000, 20001, (5, 64)).astype(np.int16)
    y, scale = plain.quantize_rows(x)
    S = scale.astype(np.float64)[:, None] / 2 ** 14
    assert np.abs(y * S - x).max() <= S.max() / 2 and np.abs(y).max() == 127
    assert plain.quantize_rows(np.zeros((1, 16), np.int16))[1].tolist() == [1]


def test_plain_linear_is_the_scaled_product():
    """Within half a unit and the 2^-28 that a factor of 29 bits may be short by."""
    g = np.random.Generator(np.random.PCG64(2))
    x, w = (g.integers(-127, 128, s).astype(np.int8) for s in ((6, 64), (1, 32, 64)))
    S = g.integers(1 << 12, 1 << 22, 6).astype(np.int32)
    mult, shift = g.integers(1, 1 << 31, (1, 32)).astype(np.int32), np.full((1, 32), 52, np.int32)
    b = g.integers(-4000, 4000, (1, 32)).astype(np.int32)
    y = np.zeros((6, 32), np.int16)
    plain.linear_scaled(x, S, w, b, mult, shift, [0, 6], None, 16, y)
    v = (x.astype(np.int64) @ w[0].T.astype(np.int64)).astype(float)
    v = v * (S[:, None] / 2 ** 14) * (mult / 2.0 ** 52)
    want = (v + b / 16).clip(-32767, 32767)
    assert (np.abs(y - want) <= 0.5 + 1 / 16 + np.abs(v) * 2.0 ** -28).all()


def test_plain_probabilities():
    """2^-30 of the true ones, and what 64 weights rounded down to 2^-30 lose."""
    g = np.random.Generator(np.random.PCG64(3))
    s = g.integers(-600, 600, 64)
    e = np.exp2(s / 64)
    p = np.array(plain.probabilities(s.tolist(), False)) / 2 ** 30
    assert np.abs(p - e / e.sum()).max() < 70 * 2.0 ** -30
    p = np.array(plain.probabilities(s.tolist(), True)) / 2 ** 30
    assert np.abs(p - e / (1 + e)).max() < 4 * 2.0 ** -30


# -------------------------------------------------------------- built kernels
@pytest.mark.parametrize("name", ["quantize_kernel", "scaled_kernel", "stream_kernel",
                                  "choose_kernel", "place_kernel", "combine_kernel",
                                  "log_probs_kernel", "log_probs_join_kernel"])
def test_no_private_memory(kernels, name):  # noqa: F811
    found = named(kernels, name)
    assert found
    bad = {k: (v[".private_segment_fixed_size"], v[".vgpr_spill_count"]) for k, v in found.items()
           if v[".private_segment_fixed_size"] or v[".vgpr_spill_count"]}
    assert not bad
