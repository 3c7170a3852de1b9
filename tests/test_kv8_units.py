"""The units that attention over an 8-bit cache sums values in (csrc/pv_kv8_units.h), compiled for the host: sums of float numbers kept by its rule against 64 bits.

Every key has weight 1 and code 448, a group of 16 keys adds 16 * f16(2^(15 + dv)) * 448.  What the rule gives has to be finite, and right: a power of two loses nothing as f16 from 2^-24 on (dv >= -39),
a group looked at in its own unit has dv = 0, and one that is dropped is 2^-64 of the largest or less, so that a sum in 32 bits of n groups is off by n * 2^-24 of itself, and n * 2^-39 for what rounds to zero."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NO_SCALE = -1000

SOURCE = r"""
#include <algorithm>
#include <math.h>
#define __device__
using std::max; using std::min;
#include "pv_kv8_units.h"
// ev: groups of exponents, four at a time; w: their weights (1 or 0); start: what the accumulator begins with, in the unit E0 (NO_SCALE: nothing)
extern "C" int walk(const int *ev, const float *w, int n, float start, int E0, float *sum, int *unit, int *passes, int *fall)
{
    float O = start;
    int E = E0, top = E0;
    *passes = 0; *fall = 0;
    for (int i = 0; i < n; i += 4) {
        int only = -1;
        for (;;) {
            const int four[4] = {ev[i], ev[i + 1], ev[i + 2], ev[i + 3]};
            int dv[4], to = E;
            const int before = only;
            kv8_next_unit(four, to, top, dv, only);
            if (before >= 0 && only != before) return 1;
            if (E != KV8_NO_SCALE) O = ldexpf(O, E - to);
            E = to;
            *fall = max(*fall, top - E);
            for (int g = 0; g < 4; ++g) {
                if (four[g] == KV8_NO_SCALE || (only >= 0 && g != only)) continue;
                if (dv[g] > 0 || (only >= 0 && dv[g] < -KV8_FALL)) return 2;
                O += w[i + g] * 16 * (float)(_Float16)ldexpf(1.f, 15 + dv[g]) * 448.f;
            }
            ++*passes;
            if (only < 0 || only == 3) break;
            ++only;
        }
    }
    *sum = O; *unit = E;
    return 0;
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    cc = shutil.which("g++") or shutil.which("clang++")
    if cc is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("units")
    (d / "units.cpp").write_text(SOURCE)
    so = str(d / "units.so")
    r = subprocess.run([cc, "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2505_01572_amd", "csrc"), "-o", so, str(d / "units.cpp")], capture_output=True, text=True)
    if r.returncode and "_Float16" in r.stderr:
        cc = "/opt/rocm/llvm/bin/clang++"
        subprocess.check_call([cc, "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2505_01572_amd", "csrc"), "-o", so, str(d / "units.cpp")])
    elif r.returncode:
        raise AssertionError(r.stderr)
    f = ctypes.CDLL(so).walk
    f.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_int] + [ctypes.c_void_p] * 4

    def go(ev, w=None, start=0.0, unit=NO_SCALE):
        ev = np.ascontiguousarray(ev, dtype=np.int32)
        w = np.ones(len(ev), np.float32) if w is None else np.ascontiguousarray(w, dtype=np.float32)
        o, E, passes, fall = ctypes.c_float(), ctypes.c_int(), ctypes.c_int(), ctypes.c_int()
        assert f(ev.ctypes.data, w.ctypes.data, len(ev), start, unit, *(ctypes.byref(x) for x in (o, E, passes, fall))) == 0
        assert np.isfinite(o.value) and 0 <= fall.value <= 64
        return o.value, E.value, passes.value
    return go


def wanted(ev, w=None):
    ev = np.asarray(ev)
    live = ev != NO_SCALE
    return float((np.where(live, 1.0, 0.0) * (1.0 if w is None else w) * 16 * 448 * 2.0 ** np.where(live, ev, 0)).sum())


def near(got, E, ev, w=None):
    want = wanted(ev, w)
    value = np.ldexp(np.float64(got), E - 15)
    assert abs(value - want) <= want * len(ev) * (2.0 ** -24 + 2.0 ** -39), (value, want)


def test_a_block_of_zeros_costs_no_pass_and_overflows_nothing(walk):
    for e in (0, -8, 40, 110, -30):
        for n in (4, 64, 4096):
            ev = [e] * n + [e, e, e, -100]
            o, E, passes = walk(ev)
            assert E == e and passes == n // 4 + 1
            near(o, E, ev)
            o, E, _ = walk([-100] * 4 + ev + [-100] * 8 + [e + 3] * 4)
            near(o, E, [-100] * 4 + ev + [-100] * 8 + [e + 3] * 4)


def test_a_sum_of_2_30_keys_holds_whatever_follows(walk):
    """The accumulator as 2^30 keys of the largest code leave it, and then groups of every kind."""
    full = float(2.0 ** 15 * 448 * 2.0 ** 30)
    r = np.random.default_rng(0)
    for e in (0, 126, -60):
        for _ in range(300):
            ev = e - r.integers(0, 130, 64)
            ev[r.random(64) < 0.2] = NO_SCALE
            o, E, _ = walk(np.maximum(ev, -1000), start=full, unit=e)
            assert o <= 2.0 ** 118 * 1.01 and np.ldexp(np.float64(o), E - 15) >= np.ldexp(full, e - 15) * (1 - 1e-5)


def test_scales_that_fall_step_by_step(walk):
    """A fall each time of less than the rule's 2^64, but more in all."""
    for step in (5, 14, 15, 20, 50, 56, 63, 64, 65):
        ev = np.repeat(100 - step * np.arange(40), 4)
        ev = ev[ev >= -126]
        o, E, _ = walk(ev)
        near(o, E, ev)
        o, E, _ = walk(np.concatenate([ev, ev[::-1], ev]))
        near(o, E, np.concatenate([ev, ev[::-1], ev]))


def test_any_exponents(walk):
    r = np.random.default_rng(1)
    for spread in (1, 13, 16, 30, 63, 66, 120, 250):
        for _ in range(100):
            ev = r.integers(-126, -126 + spread + 1, 40) + r.integers(0, 253 - spread)
            ev[r.random(40) < 0.15] = NO_SCALE
            o, E, _ = walk(ev)
            if (ev != NO_SCALE).any():
                near(o, E, ev)


def test_values_that_count_beside_larger_ones_that_do_not(walk):
    """Groups of up to 2^-63 of the largest, which has no weight: their sum is what is wanted."""
    r = np.random.default_rng(2)
    for d in (1, 10, 14, 15, 16, 30, 50, 60, 63):
        for _ in range(30):
            ev = np.full(32, -d) + 20
            w = np.ones(32)
            big = r.integers(0, 32, 3)
            ev[big], w[big] = 20, 0.0
            o, E, _ = walk(ev, w)
            near(o, E, ev, w)
