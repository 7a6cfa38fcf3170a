"""Calls on a stream of their own: whose memory their outputs are, and temporaries that are dropped
while the calls that use them are still to run."""

import numpy as np
import pytest

from oracle import core
from workloads import make_groupnorm, make_linear
from workloads.generate import INT8, INT16

pytestmark = pytest.mark.gpu

S8, S16 = 1 / 32, 1 / 4096
B, T, D, F = 3, 61, 128, 256


def _dev(a):
    import torch

    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _stream_of(t):
    """The stream whose pool of the caching allocator holds ``t``."""
    import torch

    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not in the caching allocator")


class Chain:
    def __init__(self, ipk):
        self.up_p = make_linear(D, F, 1, S16, INT16, INT16, S16)
        self.norm_p = make_groupnorm(F, 8, 2, INT16, INT16, True, S16, S16)
        self.down_p = make_linear(F, D, 3, S16, INT16, INT8, S8, S_z=S8)
        self.ipk, self.up, self.down = ipk, ipk.Linear(self.up_p), ipk.Linear(self.down_p)
        self.norm = ipk.GroupNorm(self.norm_p, max_batch=B, max_T=T)

    def __call__(self, x, z, lengths, stream):
        q = self.ipk.quantize_tokens
        h = self.norm(self.up(*q(x, stream=stream), stream=stream), lengths=lengths, stream=stream)
        return self.down(*q(h, stream=stream), z=z, stream=stream)

    def oracle(self, x, z, lengths):
        h = core.groupnorm(self.norm_p, core.token_linear(self.up_p, *core.quantize_tokens(x)), lengths)
        return core.token_linear(self.down_p, *core.quantize_tokens(h), z)

    def close(self):
        for m in (self.up, self.down, self.norm):
            m.close()


def _inputs(seed):
    rng = np.random.default_rng(seed)
    x = np.clip(np.rint(rng.normal(size=(B, T, D)) * 4096), -32767, 32767).astype(np.int16)
    return x, np.clip(np.rint(rng.normal(size=(B, T, D)) * 32), -127, 127).astype(np.int8)


def test_outputs_are_the_given_streams(gpu_lib):
    import torch

    c = Chain(gpu_lib)
    x, z = (_dev(a) for a in _inputs(0))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    q, s = gpu_lib.quantize_tokens(x, stream=st)
    h = c.up(q, s, stream=st)
    n = c.norm(h, stream=st)
    assert [_stream_of(t) for t in (q, s, h, n)] == [st.cuda_stream] * 4
    cur = torch.cuda.current_stream()
    for stream in (None, cur):
        q, s = gpu_lib.quantize_tokens(x, stream=stream)
        h = c.up(q, s, stream=stream)
        n = c.norm(h, stream=stream)
        assert [_stream_of(t) for t in (q, s, h, n)] == [cur.cuda_stream] * 4
    torch.cuda.synchronize()
    c.close()


def test_temporaries_dropped_before_their_calls_have_run(gpu_lib):
    """The chain's temporaries and its inputs are dropped while the stream is still busy with other work, and the
    current stream then allocates and fills blocks of their sizes."""
    import torch

    c = Chain(gpu_lib)
    st, cur = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.randn((2048, 2048), device="cuda")
    lengths = [T, 40, 1]
    outs, wants = [], []
    for k in range(6):
        x, z = _inputs(k)
        xd, zd = _dev(x), _dev(z)
        st.wait_stream(cur)
        with torch.cuda.stream(st):
            for _ in range(20):
                torch.mm(busy, busy)
        outs.append(c(xd, zd, lengths, st))
        wants.append(c.oracle(x, z, lengths))
        del xd, zd
        for shape, dt in (((B, T, D), torch.int16), ((B, T, D), torch.int8), ((B, T), torch.int32),
                          ((B, T, F), torch.int16), ((B, T, F), torch.int8)):
            for _ in range(3):
                torch.full(shape, 99, dtype=dt, device="cuda")
    cur.wait_stream(st)
    got = [y.cpu().numpy() for y in outs]
    for k in range(6):
        assert np.array_equal(got[k], wants[k]), k
    c.close()


def test_output_dropped_while_the_current_stream_reads_it(gpu_lib):
    """A block of the given stream goes back to it only when the current stream has read it."""
    import torch

    c = Chain(gpu_lib)
    st, cur = torch.cuda.Stream(), torch.cuda.current_stream()
    busy = torch.randn((2048, 2048), device="cuda")
    x, z = _inputs(7)
    xd, zd = _dev(x), _dev(z)
    other = _dev(_inputs(8)[0])
    want = c.oracle(x, z, None)
    kept = []
    for _ in range(4):
        st.wait_stream(cur)
        y = c(xd, zd, None, st)
        cur.wait_stream(st)
        for _ in range(20):
            torch.mm(busy, busy)
        kept.append(y.clone())
        del y
        for _ in range(3):  # allocates blocks of the dropped output's size
            c(other, zd, None, st)
    torch.cuda.synchronize()
    for k, y in enumerate(kept):
        assert np.array_equal(y.cpu().numpy(), want), k
    c.close()


def test_chain_on_a_side_stream_captured_in_a_graph(gpu_lib):
    """A captured graph that forks to a stream of the chain's own and joins again, replayed with new inputs
    and the program's own work between the replays."""
    import torch

    c = Chain(gpu_lib)
    st, lengths = torch.cuda.Stream(), [T, 1, 33]
    xs, zs = (_dev(a) for a in _inputs(0))
    out = torch.zeros_like(zs)
    c(xs, zs, lengths, None)  # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = torch.cuda.current_stream()
        st.wait_stream(cap)
        y = c(xs, zs, lengths, st)
        cap.wait_stream(st)
        out.copy_(y)
    for k in range(4):
        x, z = _inputs(20 + k)
        xs.copy_(_dev(x))
        zs.copy_(_dev(z))
        out.fill_(k)
        graph.replay()
        x2 = _dev(_inputs(30 + k)[0])
        q2, s2 = gpu_lib.quantize_tokens(x2)
        torch.cuda.synchronize()
        assert np.array_equal(out.cpu().numpy(), c.oracle(x, z, lengths)), k
        qr, sr = core.quantize_tokens(x2.cpu().numpy())
        assert np.array_equal(q2.cpu().numpy(), qr) and np.array_equal(s2.cpu().numpy(), sr), k
    del graph
    c.close()
