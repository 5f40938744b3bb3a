"""Whole numbers that do not fit the C entries' 32-bit arguments are refused by the
binding: ctypes keeps the low bits of what is wider, so that the library would be called
with another number.  On the CPU: the library's launching entries are taken away."""
import numpy as np
import pytest
import torch

from paper_2607_24981_amd import ilw, synth

i8, i16, i32 = torch.int8, torch.int16, torch.int32


class HostOnly:
    """The library without the entries that launch."""

    def __init__(self, real):
        self.real = real

    def __getattr__(self, name):
        if name == "ilw_last_error" or name.endswith("_workspace_bytes"):
            return getattr(self.real, name)

        def called(*args):
            raise AssertionError(f"{name} was called")
        return called


@pytest.fixture
def host(monkeypatch):
    monkeypatch.setattr(ilw, "_LIB", HostOnly(ilw.lib()))
    monkeypatch.setattr(ilw, "_device", lambda t, name: -1)  # where a CPU tensor says it is
    monkeypatch.setattr(ilw, "_raw_stream", lambda device: 0)
    monkeypatch.setattr(ilw, "_dev", lambda t, dtype, name: ilw.c_vp(t.data_ptr()))
    monkeypatch.setattr(ilw, "_stream", lambda: None)


def z(*shape, dtype=i8):
    return torch.zeros(*shape, dtype=dtype)


WIDE = 1 << 32
# a number that does not fit, and what its low 32 bits are
WIDER = [(5 << 30, 1 << 30), (1 << 32, 0), ((1 << 32) + 4, 4), (-(1 << 31) - 1, (1 << 31) - 1),
         (-(1 << 32) + 4, 4), (1 << 80, 0), ((1 << 63) + 4, 4)]


def refused(call, match="32 bits"):
    with pytest.raises(ilw.IlwError, match=match):
        call()


def reaches_the_library(call):
    with pytest.raises(AssertionError, match="was called"):
        call()


ROUTE = ["top_k", "groups", "top_groups", "group_best", "sigmoid", "renormalize", "weight_mult",
         "weight_shift"]


@pytest.mark.parametrize("value", [w for w, _ in WIDER])
@pytest.mark.parametrize("name", ROUTE)
def test_route(host, name, value):
    kw = {"top_k": 2}
    reaches_the_library(lambda: ilw.ilw_route(z(3, 8, dtype=i16), **kw))
    kw[name] = value
    refused(lambda: ilw.ilw_route(z(3, 8, dtype=i16), **kw))


@pytest.mark.parametrize("value", [w for w, _ in WIDER])
@pytest.mark.parametrize("name", ["mult", "shift", "skip_mult"])
def test_combine(host, name, value):
    kw = {"mult": 3, "shift": 4, "skip_mult": 5}

    def call():
        return ilw.ilw_combine(z(4, 16), z(2, 2, dtype=i32), z(2, 2, dtype=i32), skip=z(2, 16), **kw)
    reaches_the_library(call)
    kw[name] = value
    refused(call)


@pytest.mark.parametrize("value", [w for w, _ in WIDER])
def test_log_probs(host, value):
    reaches_the_library(lambda: ilw.ilw_log_probs(z(3, 8, dtype=i16), top=4))
    refused(lambda: ilw.ilw_log_probs(z(3, 8, dtype=i16), top=value))


def test_the_limits_themselves(host):
    """What fits goes on to the library, which says what it allows."""
    most, least = (1 << 31) - 1, -(1 << 31)
    x = z(3, 8, dtype=i16)
    for kw in (dict(weight_mult=most), dict(weight_mult=least), dict(weight_shift=most)):
        reaches_the_library(lambda: ilw.ilw_route(x, 2, **kw))
    for v in (most, least):
        reaches_the_library(lambda: ilw.ilw_combine(z(4, 16), z(2, 2, dtype=i32),
                                                    z(2, 2, dtype=i32), v, v, skip_mult=v))


def untouched(*shape, dtype):
    """A tensor of that many values whose memory is never touched (not even got, where
    the system counts what a program asked for: the case is skipped)."""
    try:
        return torch.empty(*shape, dtype=dtype)
    except RuntimeError as e:
        pytest.skip(f"{shape} values: {e}")


def none(*shape):
    return z(0, *shape)


# tensors whose sizes do not fit: their low bits are a call's that could be made
SIZES = {
    "quantize values": lambda: ilw.ilw_quantize_rows(untouched(1, WIDE + 16, dtype=i16)),
    "route tokens": lambda: ilw.ilw_route(z(1, 1, dtype=i16).expand(WIDE + 3, 1), 1),
    "route experts": lambda: ilw.ilw_route(untouched(1, WIDE + 8, dtype=i16), 1),
    "log_probs vocabulary": lambda: ilw.ilw_log_probs(untouched(1, WIDE + 8, dtype=i16)),
    "log_probs given": lambda: ilw.ilw_log_probs(none(8).to(i16), none(WIDE + 2).to(i32)),
    "combine values": lambda: ilw.ilw_combine(untouched(1, WIDE + 16, dtype=i8), z(1, 1, dtype=i32),
                                              z(1, 1, dtype=i32), 1, 1),
    "combine choices": lambda: ilw.ilw_combine(none(16), none(WIDE + 2).to(i32),
                                               none(WIDE + 2).to(i32), 1, 1),
    "linear inputs": lambda: ilw.ilw_linear_scaled(
        none(WIDE + 16), z(0, dtype=i32), none(WIDE + 16), None, *[z(1, dtype=i32)] * 2),
    "linear factors": lambda: ilw.ilw_linear_scaled(
        z(2, 16), z(2, dtype=i32), z(16, 16), None, *[z(1, dtype=i32).expand(WIDE + 16)] * 2),
}


@pytest.mark.parametrize("name", SIZES)
def test_sizes(host, name):
    refused(SIZES[name])


# ------------------------------------------- the operators before those, each number apart
def attention(**kw):
    p = dict(score_mult=1 << 20, score_shift=30, smax_I0=100, smax_k_inter=16, smax_k_out=8,
             smax_m_p=4, smax_s_d=-1, pv_mult=1 << 20, pv_shift=30, grid_h=2, grid_w=2, win_h=2,
             win_w=2, heads=2)
    p.update(kw)
    return ilw.ilw_attention(z(1, 4, 3 * 64), *[p.pop(k) for k in
                                                ("grid_h", "grid_w", "win_h", "win_w", "heads")], p)


def deform(entry, refs, **kw):
    p = dict(I0=100, out_mult=1 << 20, out_shift=20, mode=0, s_d=-1, k_inter=16, k_out=8, m_p=4)
    p.update(kw)
    return entry(z(1, 4, 2, 32), [[2, 2]], [0], z(1, 3, refs, dtype=i32),
                 z(1, 3, 2, 1, 4, 2, dtype=i16), z(1, 3, 2, 4), **p)


def cache():
    return ilw.KVCache(z(4, 2, 16, 64), z(4, 2, 16, 64), z(4, 2, dtype=i32), z(4, 2, dtype=i32),
                       z(1, 4, dtype=i32))


def cache_append(heads=2, max_new=1):
    return ilw.ilw_cache_append(cache(), z(1, (2 + 4) * 64), heads, z(2, dtype=i32),
                                z(1, dtype=i32), max_new)


def cache_attention(max_q=1, max_len=16, causal=True, window=0, **kw):
    p = dict(score_mult=1 << 26, score_shift=34, out_mult=1 << 30, out_shift=44)
    p.update(kw)
    return ilw.ilw_cache_attention(cache(), z(1, 2, 64), z(1, 2, dtype=i32), z(2, dtype=i32),
                                   z(1, dtype=i32), p, max_q, max_len, causal, window)


def patch_embed(**kw):
    p = dict(pos_mult_a=1, pos_mult_b=1, pos_shift=8)
    p.update(kw)
    return ilw.ilw_patch_embed(z(1, 3, 16, 16), z(16, 768), None, z(1, dtype=i32), z(1, dtype=i32),
                               z(1, 16), **p)


EARLIER = {
    "shiftmax": (lambda **kw: ilw.ilw_shiftmax(z(2, 16), **{"I0": 9, **kw}),
                 "I0 k_inter k_out m_p s_d"),
    "sdshiftgelu": (lambda **kw: ilw.ilw_sdshiftgelu(z(2, 16), **{
        "I0": 9, "out_mult": 1, "out_shift": 4, **kw}), "I0 out_mult out_shift k_inter k_out"),
    "shiftmax_ivit": (lambda **kw: ilw.ilw_shiftmax_ivit(z(2, 16), **{"I0": 9, **kw}),
                      "I0 M k_inter k_out"),
    "shiftgelu_ivit": (lambda **kw: ilw.ilw_shiftgelu_ivit(z(2, 16), **{
        "I0": 9, "out_mult": 1, "out_shift": 4, **kw}), "I0 out_mult out_shift k_inter k_out"),
    "int_layernorm": (lambda **kw: ilw.ilw_int_layernorm(
        z(2, 16), z(16, dtype=i32), z(16, dtype=i32), z(16, dtype=i32), **kw), "newton_iters"),
    "residual_add": (lambda **kw: ilw.ilw_residual_add(z(2, 16), z(2, 16), **{
        "mult_a": 1, "mult_b": 1, "shift": 4, **kw}), "mult_a mult_b shift"),
    "attention": (attention, "score_mult score_shift smax_I0 smax_k_inter smax_k_out smax_m_p "
                             "smax_s_d pv_mult pv_shift grid_h grid_w win_h win_w heads"),
    "patch_embed": (patch_embed, "patch pos_mult_a pos_mult_b pos_shift"),
    "deform_attn": (lambda **kw: deform(ilw.ilw_deform_attn, 2, **kw),
                    "I0 out_mult out_shift mode s_d k_inter k_out m_p"),
    "deform_attn_boxes": (lambda **kw: deform(ilw.ilw_deform_attn_boxes, 4, **kw), "I0 out_mult"),
    "cache_append": (cache_append, "heads max_new"),
    "cache_attention": (cache_attention, "score_mult score_shift out_mult out_shift max_q max_len "
                                         "causal window"),
}


@pytest.mark.parametrize("entry,name", [(e, n) for e, (_, names) in EARLIER.items()
                                        for n in names.split()])
def test_earlier_entries(host, entry, name):
    call = EARLIER[entry][0]
    reaches_the_library(call)
    for value, _ in WIDER:
        refused(lambda: call(**{name: value}))


def numbers(p):
    return [n for n, v in p.items() if isinstance(v, int)]


def test_parameters_of_layers(host):
    """Every number that a block and a decoder layer are made from."""
    g = np.random.Generator(np.random.PCG64(5))
    for make, p in ((ilw.DeviceBlock, synth.block_params(g, 64, 1, 64, 64)),
                    (ilw.DeviceDecoder, synth.decoder_params(g, 32, 1, 32, 1, 4))):
        make(p, "cpu")
        assert len(numbers(p)) > 20
        for name in numbers(p):
            for value, _ in WIDER:
                refused(lambda: make({**p, name: value}, "cpu"))
    block = ilw.DeviceBlock(synth.block_params(g, 64, 1, 64, 64), "cpu")
    x = z(1, 4, 64)
    refused(lambda: ilw.DeviceDecoder({**p, "ref_dims": WIDE + 2}, "cpu"))
    for i in range(4):
        a = [2, 2, 2, 2]
        a[i] += WIDE
        for call in (lambda: ilw.ilw_block_forward(block, x, *a), lambda: block.workspace_bytes(1, *a),
                     lambda: ilw.ilw_block_forward_noalloc(block, x, *a)):
            refused(call)
    for grid in ((WIDE + 2, 2), (2, WIDE + 2)):
        refused(lambda: ilw.Encoder([block], [(2, 2)], *grid, device="cpu"))
