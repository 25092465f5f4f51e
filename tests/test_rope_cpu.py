"""Rotary positions on the host (no GPU): frequencies, fixed-point angles, refusals."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from paper_2608_26523_amd import binding as B
from paper_2608_26523_amd.rotary import frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("header,names", [("vpp_rope.h", B.EXPORTED_ROPE), ("vpp_block_attn.h", B.EXPORTED_BLOCK)])
def test_header_symbols_exported(header, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(vpp_\w+)\s*\(", text)))
    assert declared == sorted(names)
    for n in names:
        assert hasattr(B.load(), n)


def test_turns():
    f = [0.0, 2 * math.pi, math.pi, 1.0, -1.0, 1e-9, 1e6, math.pi / 2]
    t = [int(x) for x in B.vpp_rope_turns(f)]
    assert t[0] == 0 and t[2] == 1 << 63 and t[7] == 1 << 62
    assert min(t[1], 2 ** 64 - t[1]) <= 1
    for x, got in zip(f, t):  # a 53-bit quotient's fraction of a turn
        want = (x / (2 * math.pi)) % 1.0 * 2.0 ** 64
        off = abs(got - want)
        assert min(off, 2.0 ** 64 - off) <= 2.0 ** 64 * max(abs(x), 1) * 2.0 ** -51, (x, got, want)


def test_frequencies():
    n = 64
    f, s = frequencies(n)
    assert s == 1 and np.allclose(f, [10000.0 ** (-2 * i / n) for i in range(n // 2)], rtol=1e-15)
    g, s = frequencies(n, scaling="linear", factor=4.0)
    assert s == 1 and np.array_equal(g, f / 4)
    g, s = frequencies(n, scaling="ntk", factor=4.0)
    assert s == 1 and g[0] == 1 and math.isclose(g[-1], f[-1] / 4, rel_tol=1e-12)
    g, s = frequencies(n, scaling="yarn", factor=4.0, original_len=4096)
    assert s == 0.1 * math.log(4) + 1
    turns = 4096 * f / (2 * math.pi)
    assert np.array_equal(g[turns > 40], f[turns > 40])
    assert np.allclose(g[turns < 0.8], f[turns < 0.8] / 4, rtol=1e-14)
    assert np.all((g <= f) & (g >= f / 4 * (1 - 1e-15)))
    g, s = frequencies(n, scaling="bands", factor=8.0, original_len=8192)
    turns = 8192 * f / (2 * math.pi)
    assert s == 1 and np.array_equal(g[turns >= 4], f[turns >= 4])
    assert np.allclose(g[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 4)
    assert np.allclose(g[mid], f[mid] * (1 / 8 + (turns[mid] - 1) / 3 * (1 - 1 / 8)), rtol=1e-12)
    for bad in (dict(scaling="other"), dict(scaling="yarn"), dict(scaling="linear", factor=0.0), dict(base=1.0),
                dict(scaling="linear", factor=math.inf), dict(scaling="yarn", original_len=10, beta_fast=1.0),
                dict(scaling="bands", original_len=10, high_factor=1.0)):
        with pytest.raises(ValueError):
            frequencies(n, **bad)
    with pytest.raises(ValueError):
        frequencies(24)


GOOD = 1 << 20  # an aligned address that no refused call reads


def _cfg(**over):
    a = dict(head_dim=128, rotary_dim=128, offset=0, interleaved=0, scale=1.0)
    a.update(over)
    return B.RopeConfig(**a)


def _rope(cfg=None, x=GOOD, xs=(1024, 128), out=2 * GOOD, os_=(1024, 128), tokens=4, heads=8, turns=GOOD, pos=GOOD):
    return B.load().vpp_rope(ctypes.byref(cfg or _cfg()), x, xs[0], xs[1], out, os_[0], os_[1], tokens, heads, turns, pos, 0, None)


@pytest.mark.parametrize("bad", [
    dict(cfg=_cfg(head_dim=130)), dict(cfg=_cfg(head_dim=8, rotary_dim=8)), dict(cfg=_cfg(head_dim=1032)),
    dict(cfg=_cfg(rotary_dim=0)), dict(cfg=_cfg(rotary_dim=24)), dict(cfg=_cfg(rotary_dim=144)),
    dict(cfg=_cfg(rotary_dim=64, offset=72)), dict(cfg=_cfg(rotary_dim=64, offset=4)), dict(cfg=_cfg(offset=-8)),
    dict(cfg=_cfg(interleaved=2)), dict(cfg=_cfg(scale=math.nan)), dict(cfg=_cfg(scale=math.inf)),
    dict(x=0), dict(x=GOOD + 2), dict(out=0), dict(out=2 * GOOD + 8), dict(turns=0), dict(turns=GOOD + 4), dict(pos=0),
    dict(pos=GOOD + 4), dict(tokens=-1), dict(heads=0), dict(xs=(1020, 128)), dict(xs=(0, 128)), dict(os_=(1024, 0)),
    dict(os_=(1024, 64)),                      # heads of the result overlap
    dict(os_=(512, 128)),                      # tokens of the result overlap
    dict(xs=(1 << 31, 128)),
    dict(out=GOOD + 1024),                     # overlaps the rows, but is not them
    dict(out=GOOD, os_=(2048, 128)),           # the rows' place with other strides
    dict(out=GOOD - 1024),
    dict(tokens=1 << 27, xs=(1024, 128), out=1 << 40),  # more units than the kernel counts
])
def test_rope_refusals(bad):
    assert _rope(**bad) == B.VPP_ERR_INVALID_ARG


def test_rope_of_nothing():
    assert _rope(tokens=0) == B.VPP_OK
    assert B.load().vpp_rope(None, GOOD, 8, 8, GOOD, 8, 8, 1, 1, GOOD, GOOD, 0, None) == B.VPP_ERR_INVALID_ARG
    for f in ([math.nan] * 8, [math.inf] + [0.0] * 7, [1.0] * 7, []):
        with pytest.raises(B.VppError):
            B.vpp_rope_turns(f)


def _append(cfg=None, q=GOOD, qs=(1024, 128), qo=2 * GOOD, qos=(1024, 128), k=3 * GOOD, v=4 * GOOD, kp=5 * GOOD, vp=6 * GOOD,
            ks=(256, 128), vs=(256, 128), kps=(16384, 256, 128), vps=(16384, 256, 128), tokens=4, hq=8, hkv=2, dv=128,
            page=64, pages=10, turns=GOOD, pos=GOOD, slots=GOOD):
    return B.load().vpp_rope_append_paged(ctypes.byref(cfg or _cfg()), q, *qs, qo, *qos, k, *ks, v, *vs, kp, *kps, vp, *vps,
                                          tokens, hq, hkv, dv, page, pages, turns, pos, slots, None)


@pytest.mark.parametrize("bad", [
    dict(cfg=_cfg(rotary_dim=8)), dict(q=0), dict(qo=0), dict(q=GOOD + 4), dict(qo=GOOD + 512), dict(qo=GOOD, qos=(2048, 128)),
    dict(qos=(1024, 32)), dict(k=0), dict(v=0), dict(kp=0), dict(vp=0), dict(k=GOOD + 2), dict(v=GOOD + 2), dict(kp=GOOD + 2),
    dict(vp=GOOD + 2), dict(ks=(100, 128)), dict(vs=(0, 128)), dict(kps=(16384, 256, 100)), dict(vps=(-8, 256, 128)),
    dict(tokens=-1), dict(hq=-1), dict(hkv=0), dict(dv=0), dict(dv=12), dict(dv=1032), dict(page=32), dict(page=96),
    dict(page=1 << 21), dict(pages=0), dict(turns=0), dict(pos=0), dict(slots=0), dict(slots=GOOD + 4),
])
def test_append_refusals(bad):
    assert _append(**bad) == B.VPP_ERR_INVALID_ARG


def test_append_of_nothing():
    assert _append(tokens=0) == B.VPP_OK


def test_wrapper_refusals_without_a_gpu():
    from paper_2608_26523_amd.rotary import Rotary
    for bad in (dict(head_dim=128, layout="other"), dict(head_dim=100), dict(head_dim=128, rotary_dim=24),
                dict(head_dim=128, rotary_dim=64, offset=68), dict(head_dim=128, freq=[1.0]),
                dict(head_dim=128, freq=[1.0] * 64, scaling="linear"), dict(head_dim=128, scale=math.nan),
                dict(head_dim=128, device="cpu")):
        with pytest.raises(ValueError):
            Rotary(**bad)
