"""Sizes that the library's arguments cannot hold are refused in the binding (no GPU): ctypes passes an
integer modulo 2^32, which could be a valid size again."""

import numpy as np
import pytest
import torch

from paper_2609_30846_amd import ipk

META = torch.device("meta")


@pytest.mark.parametrize("d", [65536 + 16, (1 << 32) + 16, 1 << 33])
@pytest.mark.parametrize("dtype", [torch.int16, torch.int32])
def test_quantize_refuses_rows_past_the_limit(d, dtype):
    with pytest.raises(ValueError, match="65536"):
        ipk.quantize_tokens(torch.empty((1, d), dtype=dtype, device=META))


class Buffer:
    """Host memory in a device tensor's place: a refused call does not touch it."""

    def __init__(self):
        self.a = np.zeros(4096, dtype=np.int8)

    def data_ptr(self):
        return (self.a.ctypes.data + 15) & ~15


class Called(Exception):
    pass


@pytest.fixture
def no_call(monkeypatch):
    class Lib:
        def __getattr__(self, name):
            raise Called(name)

    monkeypatch.setattr(ipk, "load", Lib)


WRAPS = (1 << 32) + 16, (1 << 31), -(1 << 31) - 1, 1 << 64


@pytest.mark.parametrize("n", WRAPS)
def test_the_raw_functions_refuse_what_would_wrap(no_call, n):
    b = Buffer()
    calls = [lambda: ipk.ipk_quantize_tokens(b, 1, 1, n, b, b), lambda: ipk.ipk_quantize_tokens(b, n, 1, 16, b, b),
             lambda: ipk.ipk_linear_run(1, b, b, n, None, b), lambda: ipk.ipk_groupnorm_run(1, b, None, n, 1, b),
             lambda: ipk.ipk_groupnorm_run(1, b, None, 1, n, b)]
    if abs(n) >= 1 << 63:
        calls.append(lambda: ipk.ipk_quantize_tokens(b, 1, n, 16, b, b))
    for call in calls:
        with pytest.raises(ValueError, match=str(n)):
            call()
