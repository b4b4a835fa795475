"""Pins of the 4-bit cache's oracle: the format by hand, rounding against exact
fractions, and the plain form of its workloads."""
import importlib.util
import os
from fractions import Fraction

import numpy as np
import torch

from oracle import fp4_oracle as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_values_by_hand():
    codes = np.array([[0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] * 2], np.uint8)
    v = F.values(codes, np.array([[129]], np.uint8))[0]
    half = [0, 2, 4, 6, 8, 12, 16, 24]
    assert v.tolist() == (half + [-x for x in half]) * 2
    assert np.signbit(v[8]) and not np.signbit(v[0])
    assert np.isnan(F.values(codes, np.array([[255]], np.uint8))).all()
    assert F.values(codes, np.array([[0]], np.uint8))[0, 7] == 6 * 2.0 ** -127
    assert np.array_equal(F.pack(F.unpack(codes)), codes)


def test_scales_are_the_smallest_that_hold_the_largest():
    r = np.random.default_rng(0)
    tops = np.concatenate([np.ldexp(r.uniform(0.5, 1, 300), r.integers(-160, 129, 300)),
                           [7 * 2.0 ** n for n in (-126, -3, 0, 5, 124, 125)], [6.999, 7.001, 0, 2.0 ** 127]])
    for t, s in zip(tops, F.scale_bytes(tops)):
        e = int(s) - 127
        assert -126 <= e <= 125
        assert e == 125 or Fraction(t) < 7 * Fraction(2) ** e
        assert e == -126 or Fraction(t) >= 7 * Fraction(2) ** (e - 1)
    assert F.scale_bytes(np.array([np.inf, np.nan])).tolist() == [255, 255]


def test_levels_are_the_nearest_ones():
    ties = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}
    for v, n in ties.items():
        assert F.nearest(v) == n
        assert F.nearest(np.nextafter(v, 0)) == F.nearest(v - 0.01) and F.nearest(np.nextafter(v, 9)) == F.nearest(v + 0.01)
        assert F.nearest(v - 0.01) + 1 == F.nearest(v + 0.01)
    assert F.nearest(np.arange(8)).tolist() == [0, 2, 4, 5, 6, 6, 7, 7]


def test_groups():
    r = np.random.default_rng(1)
    x = r.standard_normal((5, 3, 64)).astype(np.float32) * np.float32(2.0) ** r.integers(-20, 20, (5, 3, 1))
    x[0, 0, :32] = 0
    x[1, 1, 5] = np.nan
    x[2, 2, 40] = -np.inf
    codes, s = F.quantise(x)
    v = F.values(codes, s)
    bad = np.zeros((5, 3, 2), bool)
    bad[1, 1, 0] = bad[2, 2, 1] = True
    assert np.array_equal(s == 255, bad) and np.array_equal(np.isnan(v), np.repeat(bad, 32, -1))
    assert (codes.reshape(5, 3, 2, 16)[bad] == 0).all() and (v[0, 0, :32] == 0).all()
    unit = np.repeat(2.0 ** (s.astype(float) - 127), 32, -1)
    fine = ~np.isnan(v)
    assert (np.abs(v - x)[fine] <= unit[fine]).all() and (np.abs(v)[fine] <= 6 * unit[fine]).all()
    # what has been quantised stays as it is
    again = F.values(*F.quantise(v.astype(np.float32)))
    assert np.array_equal(again[fine], v[fine])


def _workloads():
    path = os.path.join(ROOT, "perf", "more_operators.py")
    spec = importlib.util.spec_from_file_location("more_operators", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.DEV = "cpu"
    return m


def test_plain_forms_of_the_workloads():
    m = _workloads()
    r = np.random.default_rng(2)
    x = (r.standard_normal((40, 2, 96)) * 2.0 ** r.integers(-130, 120, (40, 2, 1))).astype(np.float32)
    x[0, 0, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6.9]
    x[0, 0, 8:32] = 0
    codes, s = m._quantise(torch.from_numpy(x))
    ref, ref_s = F.quantise(x)
    assert np.array_equal(s.numpy(), ref_s)
    assert np.array_equal(F.values(codes.numpy(), s.numpy()), F.values(ref, ref_s))
    assert np.array_equal(m._exact_held(torch.from_numpy(x)).numpy(), F.values(ref, ref_s))
    c = r.integers(0, 256, (7, 48)).astype(np.uint8)
    s = r.integers(1, 240, (7, 3)).astype(np.uint8)
    assert np.array_equal(m._exact_values(torch.from_numpy(c), torch.from_numpy(s)).numpy(), F.values(c, s))
    for kind in ("token", "prompt", "chunk", "mixed"):
        for op in ("append", "attn", "read") if kind == "prompt" else ("append", "attn"):
            case = {"op": op, "dtype": "f32", "kind": kind, "B": 3, "q": 9, "low": 3, "high": 40, "Hq": 4, "Hk": 2,
                    "D": 64, "page": 8}
            out, ref = m.run(m.prepare(case, 5)), m.exact(case, 5)
            for k in ref:
                assert (out[k].double() - ref[k]).norm() <= 1e-6 * ref[k].norm()
