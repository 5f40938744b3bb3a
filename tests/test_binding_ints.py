"""Whole numbers that do not fit the C entries' 32-bit arguments are refused by the
binding: ctypes keeps the low bits of what is wider, so that the library would be called
with another number.  On the CPU: the library's launching entries are taken away."""
import pytest
import torch

from paper_2607_24981_amd import ilw

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
