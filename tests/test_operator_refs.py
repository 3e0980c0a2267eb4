"""Pins of the plain forms that the operators' GPU tests compare with."""
import os

import numpy as np

import operator_refs as ref
from oracle import snip_oracle as orc

HERE = os.path.dirname(os.path.abspath(__file__))


def test_grids_are_the_formats():
    assert ref.E4M3[126] == 448 and ref.E4M3[1] == 2.0 ** -9 and ref.E4M3[8] == 2.0 ** -6 and np.all(np.diff(ref.E4M3) > 0)
    assert list(ref.code_values(np.array([0x7E, 0x81, 0x38, 0xB8], np.uint8), True, 1, 4)[0]) == [448, -2.0 ** -9, 1, -1]
    assert list(ref.code_values(np.array([0xF1, 0x27], np.uint8), False, 1, 4)[0]) == [0.5, -6, 6, 1]


def test_nearest_agrees_with_the_oracle():
    rng = np.random.default_rng(0)
    t = np.concatenate([rng.normal(size=4000) * np.exp(rng.normal(size=4000) * 3), (ref.E4M3[:-1] + ref.E4M3[1:]) / 2, -(ref.E2M1[:-1] + ref.E2M1[1:]) / 2, [0.0, 500.0, -7.0]])
    t = t.astype(np.float32).astype(np.float64)
    for grid, fmt in ((ref.E4M3, 1), (ref.E2M1, 2)):
        want = [orc.decode_code(fmt, orc.encode(fmt, float(x))) for x in t]
        assert np.array_equal(ref.nearest(t, grid), np.asarray(want, dtype=np.float64))


def test_stochastic_rule():
    # a quarter of the way from 8 to 9: up for uniforms below 1/4
    u = np.arange(65536)
    assert np.mean(ref.stochastic(np.full(65536, 8.25), u, ref.E4M3) == 9) == 0.25
    assert np.all(ref.stochastic(np.full(65536, -448.0), u, ref.E4M3) == -448) and np.all(ref.stochastic(np.zeros(65536), u, ref.E4M3) == 0)
    assert np.all(ref.between(np.array([8.0, 9.0]), np.array([8.5, 8.5]), 1e-9, ref.E4M3)) and not ref.between(np.array([9.0]), np.array([8.4]), 1e-9, ref.E4M3)[0]


def test_generator_known_answers():
    # the published answer for counter 0; the others, whose counters are not small, through the oracle's generator
    lines = [line.split() for line in open(os.path.join(HERE, "golden", "philox4x32_10_kat.txt")) if line.strip() and not line.startswith("#")]
    seen = 0
    for f in lines:
        w = [int(x, 16) for x in f]
        c, k, out = w[:4], w[4:6], w[6:10]
        if c[0] == 0 and c[1] == 0:      # q counts from zero
            got = ref.philox(1, c[2], c[3], k[0] | k[1] << 32)
            assert [int(x[0]) for x in got] == out
            seen += 1
    assert seen >= 1
    got = ref.philox(5, 7, 0x80000001, 0x0123456789ABCDEF)
    for q in (0, 4):
        assert [int(x[q]) for x in got] == [int(x) for x in orc.philox4x32_10([q, 0, 7, 0x80000001], [0x89ABCDEF, 0x01234567])]


def test_norm_gradient_by_differences():
    rng = np.random.default_rng(1)
    x, gain, dy = rng.normal(size=(3, 24)), rng.normal(size=24), rng.normal(size=(3, 24))
    _, rstd, _ = ref.norm(x, None, gain, 1e-3)
    dx, dgain = ref.norm_bwd(dy, x, gain, rstd, None)
    e = 1e-6
    for r, c in ((0, 0), (1, 7), (2, 23)):
        d = np.zeros_like(x)
        d[r, c] = e
        num = ((dy * ref.norm(x + d, None, gain, 1e-3)[2]).sum() - (dy * ref.norm(x - d, None, gain, 1e-3)[2]).sum()) / (2 * e)
        assert abs(num - dx[r, c]) < 1e-7
    d = np.zeros(24)
    d[5] = e
    num = ((dy * ref.norm(x, None, gain + d, 1e-3)[2]).sum() - (dy * ref.norm(x, None, gain - d, 1e-3)[2]).sum()) / (2 * e)
    assert abs(num - dgain[5]) < 1e-7


def test_bf16_rounding_is_the_oracles():
    rng = np.random.default_rng(2)
    x = (rng.normal(size=5000) * np.exp(rng.normal(size=5000) * 5)).astype(np.float32)
    x = np.concatenate([x, np.float32([1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8])])
    from paper_2602_01410_b200 import workloads as wl
    assert np.array_equal(ref.bf16(x.astype(np.float64)), wl.bf16_bits_to_f32(wl.to_bf16_bits(x)).astype(np.float64))


def test_adamw_against_a_hand_worked_step():
    # first step: the direction is the gradient's sign whatever its size
    p, m, v, _ = ref.adamw(np.array([1.0]), np.array([2.0]), np.zeros(1), np.zeros(1), 0.1, 0.9, 0.99, 1e-12, 1, 0.5)
    assert abs(p[0] - (1 - 0.05 - 0.1)) < 1e-10 and abs(m[0] - 0.2) < 1e-15 and abs(v[0] - 0.04) < 1e-15
