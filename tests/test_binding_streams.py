"""Calls of the binding on a stream of their own (no GPU): whose memory an output is, and what the
allocator is told of the tensors that a call uses.

An output that is allocated as the current stream's but written on another one may still be in use by
earlier work of the current stream, and a temporary that is dropped after such a call goes
back to the current stream, which may write over it before the call has read it.  The library and torch's
streams are stood in for; the tensors have no memory.
"""

import contextlib
from types import SimpleNamespace

import pytest
import torch

from paper_2609_30846_amd import ipk

META = torch.device("meta")
CURRENT, SIDE = SimpleNamespace(cuda_stream=11), SimpleNamespace(cuda_stream=22)


@pytest.fixture
def log(monkeypatch):
    """(allocations as (stream, tensor), uses as {tensor id: streams}) of the calls of a test."""
    now, made, used = [CURRENT], [], {}

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    def allocating(make):
        def logged(*a, **k):
            t = make(*a, **k)
            made.append((now[-1], t))
            return t
        return logged

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: now[-1])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: now[-1].cuda_stream)
    for name in ("empty", "empty_like"):
        monkeypatch.setattr(torch, name, allocating(getattr(torch, name)))
    monkeypatch.setattr(torch.Tensor, "new_empty", allocating(torch.Tensor.new_empty))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: used.setdefault(id(t), []).append(s), raising=False)
    lib = SimpleNamespace(**{name: lambda *a: 0 for name, _, _ in ipk.SIGNATURES})
    monkeypatch.setattr(ipk, "load", lambda: lib)
    return SimpleNamespace(made=made, used=used)


def _of(cls, **attrs):
    m = cls.__new__(cls)
    m.handle, m._dev, m.device, m._index = None, META, META, 0
    for k, v in attrs.items():
        setattr(m, k, v)
    return m


def _streams(log, y):
    """The streams current in the allocations (one may go through another) that returned ``y``."""
    return {s.cuda_stream for s, t in log.made if t is y}


def _meta(*shape, dtype=torch.int8):
    return torch.empty(shape, dtype=dtype, device=META)


def _calls():
    """(name, call taking keyword arguments, its inputs, name and value of a given output)"""
    lin = _of(ipk.Linear, d_in=32, d_out=48, dtype=torch.int16)
    q, s, z = _meta(4, 32), _meta(4, dtype=torch.int32), _meta(4, 48, dtype=torch.int16)
    yield "Linear", lambda **k: lin(q, s, z=z, **k), (q, s, z), "y", _meta(4, 48, dtype=torch.int16)
    gn = _of(ipk.GroupNorm, d_model=32, max_batch=2, max_T=8, in_dtype=torch.int16, out_dtype=torch.int8)
    h = _meta(2, 8, 32, dtype=torch.int16)
    yield "GroupNorm", lambda **k: gn(h, **k), (h,), "x", _meta(2, 8, 32)
    v = _meta(2, 8, 64)
    ln, ffn, conv = _of(ipk.LayerNorm, d_model=64), _of(ipk.FeedForward, d_model=64), _of(ipk.ConvModule, d_model=64)
    yield "LayerNorm", lambda **k: ln(v, **k), (v,), "x", _meta(2, 8, 64)
    yield "FeedForward", lambda **k: ffn(v, **k), (v,), "z_out", _meta(2, 8, 64)
    yield "ConvModule", lambda **k: conv(v, **k), (v,), "z_out", _meta(2, 8, 64)
    att, pos = _of(ipk.RelPosAttn, d_model=64), _meta(15, 64)
    yield "RelPosAttn", lambda **k: att(v, pos, **k), (v, pos), "y", _meta(2, 8, 64)
    yield "RelPosAttn.residual", lambda **k: att.residual(v, pos, **k), (v, pos), "z2", _meta(2, 8, 64)


CALLS = {c[0]: c[1:] for c in _calls()}


@pytest.mark.parametrize("name", CALLS)
def test_an_output_is_its_own_streams(log, name):
    call, inputs, _, _ = CALLS[name]
    y = call(stream=SIDE)
    assert _streams(log, y) == {SIDE.cuda_stream}
    # the inputs stay until the call has run, the output until the caller's current stream has read it
    assert all(SIDE in log.used.get(id(t), []) for t in inputs) and CURRENT in log.used[id(y)]


@pytest.mark.parametrize("name", CALLS)
def test_a_given_output_stays_until_the_call_has_run(log, name):
    call, inputs, out, value = CALLS[name]
    log.made.clear()
    assert call(stream=SIDE, **{out: value}) is value
    assert not log.made and all(SIDE in log.used.get(id(t), []) for t in inputs + (value,))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("stream", [None, CURRENT])
def test_the_current_stream_needs_nothing(log, name, stream):
    y = CALLS[name][0](stream=stream)
    assert _streams(log, y) == {CURRENT.cuda_stream} and not log.used


def test_copies_of_intermediates(log):
    for call in (lambda: _of(ipk.RelPosAttn).intermediate(0, (4, 64), stream=SIDE),
                 lambda: _of(ipk.FeedForward, d_model=64, d_ff=256).intermediate(ipk.IPK_FFN_X, 4, stream=SIDE),
                 lambda: _of(ipk.ConvModule, d_model=64).intermediate(ipk.IPK_CONV_V, 1, 4, stream=SIDE)):
        y = call()
        assert _streams(log, y) == {SIDE.cuda_stream} and CURRENT in log.used[id(y)]


def test_kept_position_projection(log):
    pos = _meta(15, 64)
    _of(ipk.RelPosAttn, d_model=64).cache_positions(pos, stream=SIDE)
    assert log.used[id(pos)] == [SIDE]
    x, y = _meta(2, 8, 64), _meta(2, 8, 64)
    _of(ipk.RelPosAttn, d_model=64).run_noalloc(x, pos, y=y, stream=SIDE)
    assert log.used[id(x)] == log.used[id(y)] == [SIDE]
