"""Constants of the linear layer and the group normalization that do not fit their C types are refused
in the binding (no GPU), not taken modulo 2^32 or rounded to other values."""

from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2609_30846_amd import ipk
from workloads import make_groupnorm, make_linear
from workloads.generate import INT8, INT16


class Created(Exception):
    pass


@pytest.fixture(autouse=True)
def no_gpu(monkeypatch):
    """Weights stay on the host, and create raises Created with the descriptor."""
    class Device:
        def __init__(self, dev):
            pass

        def __enter__(self):
            pass

        def __exit__(self, *a):
            pass

    def create(desc):
        raise Created(desc)

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(ipk, "ipk_linear_create", create)
    monkeypatch.setattr(ipk, "ipk_groupnorm_create", create)


def _linear(**over):
    p = make_linear(32, 4, 1, 1 / 4096, INT16, INT8, 1 / 32, S_z=1 / 32)
    return SimpleNamespace(**{**vars(p), **over})


def _norm(**over):
    p = make_groupnorm(32, 4, 2, INT16, INT8, True, 1 / 4096, 1 / 32)
    return SimpleNamespace(**{**vars(p), **over})


@pytest.mark.parametrize("over", [
    dict(w=np.full((4, 32), 128)), dict(w=np.full((4, 32), -129, dtype=np.int16)), dict(w=np.full((4, 32), 0.5)),
    dict(w=np.full((4, 32), np.nan)), dict(mult=np.full(4, (1 << 32) + 5)), dict(mult=[1, 2, 3, 1 << 31]),
    dict(mult=[1, 2, 3, 1 << 80]), dict(bias=np.full(4, 1 << 63, dtype=np.uint64)), dict(bias=[0, 0, 0, 2.5]),
    dict(mult=np.zeros(5, dtype=np.int32)), dict(shift=(1 << 32) + 40), dict(m_z=1 << 32), dict(out_type=(1 << 32) + 1),
])
def test_linear_refuses(over):
    with pytest.raises(ValueError):
        ipk.Linear(_linear(**over), device="cpu")


@pytest.mark.parametrize("over", [
    dict(gn_mult=np.full(32, (1 << 32) + 5)), dict(gn_mult=np.full(32, 1.25)), dict(gn_bias=np.full(32, 1 << 63, dtype=np.uint64)),
    # eps of 1e-5 on a grid of 1e-5 in 2^-16 of its squared steps
    dict(eps=round(1e-5 * 65536 / 1e-10)), dict(gn_shift=(1 << 32) + 3), dict(sw_qc=1 << 32), dict(sw_q1=1 << 64),
    dict(m_sw=(1 << 32) + 1), dict(shift_sw=(1 << 32) + 40), dict(d_model=(1 << 32) + 32), dict(n_groups=(1 << 32) + 4),
])
def test_groupnorm_refuses(over):
    with pytest.raises(ValueError):
        ipk.GroupNorm(_norm(**over), max_batch=1, max_T=8, device="cpu")


@pytest.mark.parametrize("max_batch,max_T", [((1 << 32) + 1, 8), (1, (1 << 32) + 8)])
def test_groupnorm_refuses_limits(max_batch, max_T):
    with pytest.raises(ValueError):
        ipk.GroupNorm(_norm(), max_batch=max_batch, max_T=max_T, device="cpu")


def test_other_types_of_the_same_values_are_taken():
    """As before: lists, wider integers and whole floats."""
    for over in ({}, dict(mult=[1, 2, 3, (1 << 31) - 1]), dict(w=np.full((4, 32), -128, dtype=np.int64)), dict(bias=None),
                 dict(w=np.full((4, 32), 5.0)), dict(bias=np.array([0, -(1 << 59), 1 << 59, 7], dtype=object))):
        with pytest.raises(Created) as e:
            ipk.Linear(_linear(**over), device="cpu")
        d = e.value.args[0]
        assert (d.d_in, d.d_out, bool(d.bias)) == (32, 4, over.get("bias", True) is not None)
    with pytest.raises(Created) as e:
        ipk.GroupNorm(_norm(gn_mult=np.full(32, -(1 << 23), dtype=np.int64)), max_batch=1, max_T=8, device="cpu")
    assert (e.value.args[0].max_batch, e.value.args[0].max_T) == (1, 8)
