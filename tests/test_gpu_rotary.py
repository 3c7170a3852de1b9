"""Rotary positions against the definition in 64 bits (tests/kv16_ref.py).

The angle's cosine and sine are off by at most 6 * 2^-24 of the amplitude: the reduced angle, at most pi / 4, by three roundings (2.4 * 2^-24), the series by two, the amplitude by one.  A turned number is
a c - b s: that, times |a| + |b|, and two roundings of as much, together 2^-21 amplitude (|a| + |b|), and half a step of the output's type.  The angle itself is made in 64 bits: a position's product
with its frequency is off by 2^-53 of it, here and in the oracle: 2^-51 |position| (|a| + |b|) more."""
import math

import numpy as np
import pytest
import torch

import kv16_ref as ref

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def pv():
    assert torch.cuda.is_available()
    import paper_2505_01572_amd as pv
    return pv


def frequencies(base, part):
    return [base ** (-2 * i / part) for i in range(part // 2)]


def check(got, x, positions, freq, part, interleaved, amplitude=1.0):
    x = x.double().cpu().numpy()
    want = ref.turned(x, positions, freq, part, interleaved, amplitude)
    size = np.zeros_like(x)
    i = np.arange(part // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + part // 2)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    far = np.abs(np.asarray(positions, dtype=np.float64))[:, None, None]
    bound = torch.finfo(got.dtype).eps / 2 * np.abs(want) + (2.0 ** -21 + 2.0 ** -51 * far) * abs(amplitude) * size + torch.finfo(got.dtype).tiny
    worst = (np.abs(got.double().cpu().numpy() - want) / bound).max()
    assert worst <= 1, worst
    assert np.array_equal(got.double().cpu().numpy()[..., part:], x[..., part:])


CASES = [(1, 1, 16, 16), (3, 2, 48, 32), (1, 32, 128, 128), (7, 5, 64, 16), (33, 3, 96, 48), (2, 70, 128, 64), (5, 1, 256, 256), (2, 2, 1024, 1024), (300, 4, 64, 64), (17, 1, 80, 16)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,heads,hd,part", CASES)
def test_rotate(pv, rows, heads, hd, part, dtype, interleaved):
    r = np.random.default_rng(rows * 1000 + hd)
    x = torch.from_numpy(r.normal(size=(rows, heads, hd))).to(TYPES[dtype]).cuda()
    positions = r.integers(0, 200000, rows).astype(np.int32)
    positions[0] = 0
    rot = pv.Rotary(hd, rotary_dim=part, base=10000.0, interleaved=interleaved)
    got = rot.rotate(x, torch.from_numpy(positions).cuda())
    assert got.shape == x.shape and got.dtype == x.dtype and got.is_contiguous()
    check(got, x, positions, frequencies(10000.0, part), part, interleaved)
    assert torch.equal(got[0], x[0])                                      # position 0


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions(pv, interleaved):
    positions = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, -1, 1, 1000003, -77777, 2 ** 24 + 1], dtype=np.int32)
    x = torch.randn(len(positions), 2, 64, device="cuda")
    got = pv.Rotary(64, base=500000.0, interleaved=interleaved).rotate(x, torch.from_numpy(positions).cuda())
    check(got, x, positions, frequencies(500000.0, 64), 64, interleaved)


def test_every_eighth_of_a_turn(pv):
    """Angles at the borders where the reduction changes, and beside them."""
    turns = torch.tensor([1 / 8, 1 / 4, 3 / 8, 1 / 2, 1 / 8 + 2.0 ** -40, 1 / 8 - 2.0 ** -40, 1.0, 1 / 16], dtype=torch.float64, device="cuda")
    positions = np.arange(-40, 40, dtype=np.int32)
    x = torch.randn(80, 1, 16, device="cuda")
    rot = pv.Rotary(16, turns=turns, amplitude=1.25)
    got = rot.rotate(x, torch.from_numpy(positions).cuda())
    check(got, x, positions, [2 * math.pi * float(t) for t in turns], 16, False, 1.25)


SCALED = [{"kind": "linear", "factor": 4.0}, {"kind": "base", "factor": 8.0}, {"kind": "turns", "factor": 8.0, "original": 8192, "low": 1.0, "high": 4.0},
          {"kind": "ramp", "factor": 16.0, "original": 4096, "slow": 1.0, "fast": 32.0}, {"kind": "ramp", "factor": 2.0, "original": 100, "slow": 1.0, "fast": 30.0, "amplitude": 0.75}]


@pytest.mark.parametrize("scaling", SCALED, ids=[s["kind"] + str(s.get("amplitude", "")) for s in SCALED])
def test_scaled_frequencies(pv, scaling):
    n, base, s, kind = 64, 500000.0, scaling["factor"], scaling["kind"]
    freq, amplitude = frequencies(base, n), 1.0
    if kind == "linear":
        freq = [f / s for f in freq]
    elif kind == "base":
        freq = frequencies(base * s ** (n / (n - 2)), n)
        assert math.isclose(freq[-1], frequencies(base, n)[-1] / s)       # the slowest pair
    else:
        out = []
        for i, f in enumerate(freq):
            if kind == "turns":
                keep = (scaling["original"] * f / (2 * math.pi) - scaling["low"]) / (scaling["high"] - scaling["low"])
            else:
                def place(turns):
                    return n * math.log(scaling["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))
                lo, hi = max(math.floor(place(scaling["fast"])), 0), min(math.ceil(place(scaling["slow"])), n - 1)
                keep = 1 - (i - lo) / max(hi - lo, 0.001)
            keep = min(max(keep, 0.0), 1.0)
            out.append(keep * f + (1 - keep) * f / s)
        freq = out
        if kind == "ramp":
            amplitude = scaling.get("amplitude", 0.1 * math.log(s) + 1)
    positions = np.array([0, 1, 5, 4095, 8192, 70001, 131071], dtype=np.int32)
    x = torch.randn(7, 3, 128, device="cuda")
    got = pv.Rotary(128, rotary_dim=n, base=base, scaling=scaling).rotate(x, torch.from_numpy(positions).cuda())
    check(got, x, positions, freq, n, False, amplitude)


def test_strides_and_in_place(pv):
    """Heads before rows, a slice of a fused projection, results over the inputs and into another layout."""
    fused = torch.randn(21, 6 * 64, dtype=torch.bfloat16, device="cuda")
    x = fused[:, 128:320].view(21, 3, 64)
    p = torch.arange(21, dtype=torch.int32, device="cuda") * 3
    rot = pv.Rotary(64, rotary_dim=32)
    want = rot.rotate(x.contiguous(), p)
    before = fused.clone()
    into = torch.full((3, 21, 64), 7.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert rot.rotate(x, p, out=into) is into and torch.equal(into, want) and torch.equal(fused, before)
    assert torch.equal(rot.rotate(into.contiguous().transpose(0, 1).contiguous().transpose(0, 1), p), rot.rotate(want, p))
    rot.rotate(x, p, out=x)
    assert torch.equal(x, want)
    rest = torch.ones(384, dtype=torch.bool, device="cuda")
    rest[128:320] = False
    assert torch.equal(fused[:, rest], before[:, rest])                   # nothing beside the rows
    assert rot.rotate(x[:0], p[:0]).shape == (0, 3, 64) and rot.rotate(x[:, :0], p).shape == (21, 0, 64)


def test_not_finite_numbers_stay_with_their_pairs(pv):
    x = torch.randn(4, 2, 64, device="cuda")
    p = torch.tensor([3, 9, 100, 5], dtype=torch.int32, device="cuda")
    rot = pv.Rotary(64)
    clean = rot.rotate(x, p)
    x[1, 1, 7], x[2, 0, 40] = float("nan"), float("inf")
    got = rot.rotate(x, p)
    touched = torch.zeros_like(x, dtype=torch.bool)
    touched[1, 1, [7, 39]] = touched[2, 0, [8, 40]] = True
    assert torch.equal(got[~touched], clean[~touched]) and not torch.isfinite(got[touched]).any()


def test_captured_and_on_another_stream(pv):
    x, p = torch.randn(9, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.arange(9, dtype=torch.int32, device="cuda")
    rot, out = pv.Rotary(128), torch.empty(9, 4, 128, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rot.rotate(x, p, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, rot.rotate(x, p))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rot.rotate(x, p, out=out)
    for i in range(3):
        x.copy_(torch.randn(9, 4, 128)); p.add_(1000)
        graph.replay()
        assert torch.equal(out, rot.rotate(x, p))


def test_more_rows_than_a_launch_shares(pv):
    """Sizes at which the heads are shared otherwise, and offsets past 2^31 bytes."""
    x = torch.randn(3000, 40, 64, dtype=torch.float16, device="cuda")
    p = torch.randint(0, 9999, (3000,), dtype=torch.int32, device="cuda")
    rot = pv.Rotary(64)
    got = rot.rotate(x, p)
    for r in (0, 1, 1499, 2999):
        assert torch.equal(got[r:r + 1], rot.rotate(x[r:r + 1].contiguous(), p[r:r + 1].contiguous()))
    wide = torch.empty(3, 400_000_000, dtype=torch.bfloat16, device="cuda")
    y = wide[:, :128].view(3, 2, 64)
    y.copy_(x[:3, :2])
    assert torch.equal(rot.rotate(y, p[:3].contiguous()), rot.rotate(y.contiguous(), p[:3].contiguous()))
