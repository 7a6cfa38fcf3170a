"""The oracle's operators for activations without a calibrated grid under AddressSanitizer and
UndefinedBehaviorSanitizer, as test_oracle_sanitize.py has the other entry points: the types' lowest
values, constants at the ends of their ranges, ragged lengths and single frames, every error
fatal, and the outputs of the ordinary build byte for byte."""

import os
import subprocess
import sys
import textwrap

import numpy as np
import pytest

from oracle import build as oracle_build
from oracle import core
from tests.test_oracle_sanitize import _runtime
from workloads import make_groupnorm, make_linear
from workloads.generate import INT8, INT16, INT32, TYPE_BITS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NP = (np.int8, np.int16, np.int32)
GRID = (1 / 32, 1 / 4096, 2.0 ** -16)


def _cases():
    """(label, function of no arguments giving a list of arrays)"""
    rng = np.random.default_rng(3)
    out = []
    for t in (INT16, INT32):
        lim = 2 ** (TYPE_BITS[t] - 1)
        x = rng.integers(-lim, lim, (5, 32)).astype(NP[t])
        x[0], x[1], x[2] = 0, -lim, lim - 1
        x[3] = np.where(np.arange(32) == 5, -lim, 1)
        out.append((f"quantize/{t}", lambda x=x: list(core.quantize_tokens(x))))
    for t, residual in ((INT8, True), (INT16, True), (INT32, False)):
        lim = 2 ** (TYPE_BITS[t] - 1)
        for K, N, shift in ((16, 3, 32), (1040, 5, 62)):
            p = make_linear(K, N, 1, GRID[INT16], INT16, t, GRID[t], S_z=GRID[t] if residual else None)
            p.mult, p.shift, p.m_z = np.full(N, 2 ** 31 - 1, dtype=np.int32), shift, 2 ** 29 - 1
            p.bias = np.full(N, 2 ** 60 - 1)
            p.bias[0] = -p.bias[0]
            p.w[0], q = -128, np.full((4, K), -128, dtype=np.int8)
            s = np.array([2 ** 31 - 1, -2 ** 31, 0, 1], dtype=np.int32)
            z = np.full((4, N), -lim).astype(NP[t]) if residual else None
            out.append((f"linear/{t}/{K}", lambda p=p, q=q, s=s, z=z: [core.token_linear(p, q, s, z)]))
    swishes = (((1 << 20) - 1, -(1 << 38), 200, 62), (0, -(1 << 30), 131076, 33), ((1 << 20) - 1, (1 << 45) - 1, 0, 1))
    for t in (INT8, INT16):
        lim = 2 ** (TYPE_BITS[t] - 1)
        for k, (q_c, q_1, m, shift) in enumerate(swishes):
            p = make_groupnorm(32, 4, 2, t, INT16, True, GRID[t], GRID[INT16])
            p.gn_mult = np.where(np.arange(32) % 2, (1 << 24) - 1, -(1 << 24) + 1).astype(np.int32)
            p.gn_bias = np.where(np.arange(32) % 3, (1 << 56) - 1, -(1 << 56) + 1)
            p.gn_shift, p.eps = (1, 62, 30)[k], (1, 2 ** 31 - 1, 7)[k]
            p.sw_qc, p.sw_q1, p.m_sw, p.shift_sw = q_c, q_1, m, shift
            z = rng.integers(-lim, lim, (3, 9, 32)).astype(NP[t])
            z[0], z[1, :, :8] = -lim, lim - 1
            out.append((f"groupnorm/{t}/{k}", lambda p=p, z=z: [core.groupnorm(p, z, [9, 4, 1]), core.groupnorm(p, z)]))
    return out


def test_operators_clean_under_asan_and_ubsan(tmp_path):
    asan, ubsan = _runtime("libasan.so"), _runtime("libubsan.so")
    if asan is None or ubsan is None:
        pytest.skip("gcc sanitizer runtimes are not installed")
    so = str(tmp_path / "libipk_oracle_san.so")
    subprocess.run(["gcc", "-O1", "-g", "-std=c11", "-fPIC", "-shared", "-fopenmp", "-fno-omit-frame-pointer",
                    "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-o", so, oracle_build.SRC],
                   check=True)
    cases = _cases()
    np.savez(tmp_path / "ref.npz", **{f"y{i}_{j}": y for i, (_, f) in enumerate(cases) for j, y in enumerate(f())})
    child = textwrap.dedent(f"""
        import sys
        sys.path.insert(0, {ROOT!r})
        import numpy as np
        from oracle import build as oracle_build
        oracle_build.LIB = {so!r}
        from tests import test_oracle_operators_sanitize as t
        from oracle import core
        assert core.lib()._name == {so!r}, core.lib()._name
        ref = np.load({str(tmp_path / 'ref.npz')!r})
        for i, (label, f) in enumerate(t._cases()):
            for j, y in enumerate(f()):
                assert np.array_equal(y, ref[f"y{{i}}_{{j}}"]), label
            print("sanitized oracle ok:", label, flush=True)
    """)
    env = dict(os.environ, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", OMP_NUM_THREADS="2")
    r = subprocess.run([sys.executable, "-c", child], capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert r.stdout.count("sanitized oracle ok") == len(cases)
