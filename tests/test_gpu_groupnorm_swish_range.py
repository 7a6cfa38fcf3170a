"""Group normalization with Swish constants whose products lie between 2^62 and 2^63, against the oracle."""

import numpy as np
import pytest

from oracle import core
from workloads import make_groupnorm
from workloads.generate import INT8, INT16

pytestmark = pytest.mark.gpu

GRID = {INT8: 1 / 32, INT16: 1 / 4096}


def _run(ipk, p, z, lengths):
    import torch

    mod = ipk.GroupNorm(p, max_batch=z.shape[0], max_T=z.shape[1])
    x = mod(torch.from_numpy(z).cuda(), lengths=lengths)
    torch.cuda.synchronize()
    bad = np.argwhere(x.cpu().numpy() != core.groupnorm(p, z, lengths))
    assert bad.size == 0, (tuple(bad[0]), len(bad))
    mod.close()


def _input(rng, B, T, d, tin):
    lim = (127, 32767)[tin]
    z = np.clip(np.rint(rng.normal(size=(B, T, d)) * lim / 8), -lim, lim)
    z[:, 0, ::7] = lim  # values whose Swish is among the largest
    z[:, 0, 1::7] = -lim - 1
    return z.astype((np.int8, np.int16)[tin])


@pytest.mark.parametrize("tin", [INT8, INT16])
@pytest.mark.parametrize("tout,shift_sw", [(INT8, 54), (INT16, 47)])
@pytest.mark.parametrize("B,T,d,G,lengths", [
    # one kernel, with one group and with several a workgroup, two kernels, three
    (2, 100, 256, 8, [100, 33]), (2, 60, 96, 12, None), (1, 900, 256, 2, [899]), (1, 1000, 512, 64, None)])
def test_multipliers_of_17_bits(gpu_lib, B, T, d, G, lengths, tin, tout, shift_sw):
    print(f"[groupnorm] B={B} T={T} d={d} G={G} {tin}->{tout} m_sw=130023", flush=True)
    unit = 1 / 8192
    p = make_groupnorm(d, G, 3, tin, tout, True, GRID[tin], GRID[tout], S_h=unit)
    p.sw_qc, p.sw_q1, p.m_sw, p.shift_sw = int(2.4632 / unit), int(-1 / (0.1240 * unit * unit)) - 1, 130023, shift_sw
    _run(gpu_lib, p, _input(np.random.default_rng(T), B, T, d, tin), lengths)


@pytest.mark.parametrize("tin", [INT8, INT16])
@pytest.mark.parametrize("q_c,q_1,m_sw,shift_sw", [(0, -(1 << 30), 131076, 33), (0, -(1 << 30), 131074, 48),
                                                   # negative products of 0.73 and 0.93 of 2^63: 32767 (q_c - 32767)^2 m_sw
                                                   ((1 << 20) - 1, -(1 << 38), 200, 62),
                                                   ((1 << 20) - 1, 0, 254, 48)])
def test_products_next_to_the_limit(gpu_lib, q_c, q_1, m_sw, shift_sw, tin):
    print(f"[groupnorm] limit q_c={q_c} q_1={q_1} m_sw={m_sw} shift={shift_sw} {tin}", flush=True)
    rng = np.random.default_rng(m_sw)
    p = make_groupnorm(96, 6, 4, tin, INT16, True, GRID[tin], GRID[INT16], S_h=1 / 8192)
    p.sw_qc, p.sw_q1, p.m_sw, p.shift_sw = q_c, q_1, m_sw, shift_sw
    _run(gpu_lib, p, _input(rng, 2, 40, 96, tin), [40, 7])
