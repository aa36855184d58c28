"""Host side of the operators that compute with the payload: rotary frequencies, struct layouts, refusals without a device."""
from __future__ import annotations

import ctypes as C
import math

import pytest

import __graft_entry__ as entry
from paper_2607_10987_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    entry.build()


def test_struct_sizes_match_the_header():
    assert C.sizeof(B.aaf_kv_attn) == 48 and C.sizeof(B.aaf_kv_store_desc) == 104 and C.sizeof(B.aaf_kv_rope_scaling) == 40


def test_null_pool_is_rejected():
    one = (C.c_int32 * 1)(0)
    assert B.aaf_kv_reserve(None, 1, one, one, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_store(None, 0, None, 1, one, one, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_attend(None, 0, None, 1, one, None, None, None, None, None, 0, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_attn_mass(None, 0, None, 1, one, None, None, None, None, None, 0, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_prune(None, 0, None, 1, 0, 0, None, None, None, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_attend_workspace_bytes(None) == 0


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0)])
def test_plain_frequencies(rot, base):
    f, m = B.rope_freqs(rot, base)
    assert m == 1.0 and len(f) == rot // 2
    for i, x in enumerate(f):
        assert math.isclose(x, base ** (-2.0 * i / rot), rel_tol=1e-14)


def test_linear_and_base_scaling():
    f, _ = B.rope_freqs(64)
    lin, m = B.rope_freqs(64, scaling=B.AAF_ROPE_LINEAR, factor=4.0)
    assert m == 1.0 and all(math.isclose(a, b / 4, rel_tol=1e-14) for a, b in zip(lin, f))
    ntk, _ = B.rope_freqs(64, scaling=B.AAF_ROPE_BASE, factor=4.0)
    assert ntk[0] == f[0] == 1.0 and math.isclose(ntk[-1], f[-1] / 4, rel_tol=1e-12)
    assert all(b / 4 <= a * (1 + 1e-12) and a <= b * (1 + 1e-12) for a, b in zip(ntk, f))


def test_wavelength_scaling():
    f, _ = B.rope_freqs(128, 500000.0)
    g, m = B.rope_freqs(128, 500000.0, B.AAF_ROPE_WAVELENGTH, factor=8.0, low=1.0, high=4.0, orig_context=8192.0)
    assert m == 1.0
    kinds = set()
    for a, b in zip(f, g):
        turns = 8192.0 * a / (2 * math.pi)
        if turns >= 4:
            assert b == a
            kinds.add("kept")
        elif turns <= 1:
            assert math.isclose(b, a / 8, rel_tol=1e-14)
            kinds.add("divided")
        else:
            w = (turns - 1) / 3
            assert math.isclose(b, (1 - w) * a / 8 + w * a, rel_tol=1e-12)
            kinds.add("blend")
    assert kinds == {"kept", "divided", "blend"}


def test_ramp_scaling():
    f, _ = B.rope_freqs(128)
    g, m = B.rope_freqs(128, 10000.0, B.AAF_ROPE_RAMP, factor=16.0, low=1.0, high=32.0, orig_context=4096.0)
    assert math.isclose(m, 0.1 * math.log(16) + 1, rel_tol=1e-6)
    index = lambda turns: 128 * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))
    lo, hi = math.floor(index(32)), math.ceil(index(1))
    for i, (a, b) in enumerate(zip(f, g)):
        w = min(1.0, max(0.0, (i - lo) / (hi - lo)))
        assert math.isclose(b, w * a / 16 + (1 - w) * a, rel_tol=1e-12)
    assert g[0] == f[0] and math.isclose(g[-1], f[-1] / 16, rel_tol=1e-12)


def test_frequency_refusals():
    for kw in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=8, base=1.0), dict(rot_dim=8, base=math.nan),
               dict(rot_dim=8, scaling=9), dict(rot_dim=8, scaling=-1), dict(rot_dim=8, scaling=B.AAF_ROPE_LINEAR, factor=0.5),
               dict(rot_dim=8, scaling=B.AAF_ROPE_LINEAR, factor=math.inf), dict(rot_dim=2, scaling=B.AAF_ROPE_BASE, factor=2.0),
               dict(rot_dim=8, scaling=B.AAF_ROPE_WAVELENGTH, factor=2.0, low=4.0, high=1.0, orig_context=100.0),
               dict(rot_dim=8, scaling=B.AAF_ROPE_RAMP, factor=2.0, low=1.0, high=32.0, orig_context=0.0)):
        with pytest.raises(ValueError):
            B.rope_freqs(**kw)
    out = (C.c_double * 4)()
    assert B.aaf_kv_rope_freqs(8, 10000.0, B.AAF_ROPE_LINEAR, None, out, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_rope_freqs(8, 10000.0, B.AAF_ROPE_NONE, None, None, None) == B.AAF_ERR_INVALID_ARG
    assert B.aaf_kv_rope_freqs(8, 10000.0, B.AAF_ROPE_NONE, None, out, None) == 0
