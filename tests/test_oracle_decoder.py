"""The 64-bit oracle of the operators around the GEMVs against worked values and brute force, and
planted mistakes that its pins reject."""
import numpy as np
import pytest

from oracle import decoder as od


def test_e4m3_and_e2m1_tables():
    v = od.e4m3_values()
    assert v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7e] == 448.0
    assert np.isnan(v[0x7f]) and np.isnan(v[0xff]) and v[0xb8] == -1.0
    assert np.all(np.diff(v[:127]) > 0)
    assert list(od.e2m1_values()[:8]) == [0, .5, 1, 1.5, 2, 3, 4, 6]


def test_fp4_rounds_to_nearest_ties_to_even():
    x = np.zeros(32)
    x[:16] = [6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, 0.26, 0.74, 5.01, 4.99, -6, -5]
    codes, scale = od.encode(x[None], od.FP4)
    got = od.decode(codes, scale, od.FP4)[0]
    assert scale[0, 0] == 127
    assert list(got[:16]) == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, .5, .5, 6, 4, -6, -4]


@pytest.mark.parametrize("fmt,limit,e_max", [(od.FP8, 448.0, 7), (od.FP4, 6.0, 13)])
def test_power_of_two_is_the_smallest_that_holds_the_block(fmt, limit, e_max):
    for top, e in [(limit, 0), (np.nextafter(np.float32(limit), np.float32(1e9)), 1), (limit / 2, -1), (0.0, -14),
                   (limit * 2.0 ** -14, -14), (1e-30, -14), (limit * 2.0 ** e_max, e_max), (3e38, e_max),
                   (np.inf, e_max)]:
        x = np.zeros((1, 32))
        x[0, 5] = -top
        codes, scale = od.encode(x, fmt)
        assert int(scale[0, 0]) - 127 == e, top
        if top >= limit * 2.0 ** e_max:  # saturated
            assert od.decode(codes, scale, fmt)[0, 5] == -limit * 2.0 ** e_max


def test_every_representable_value_is_kept_and_exact_in_fp16():
    for fmt, table in ((od.FP8, od.e4m3_values()[:127]), (od.FP4, od.e2m1_values()[:8])):
        limit, e_max = (448.0, 7) if fmt == od.FP8 else (6.0, 13)
        for e in (-14, -3, 0, e_max):
            vals = table * 2.0 ** e
            for i in range(0, len(vals), 31):
                x = np.zeros(32)
                part = vals[i:i + 31]
                x[:len(part)], x[31] = part, limit * 2.0 ** e
                got = od.decode(*od.encode(x[None], fmt), fmt)[0]
                assert np.array_equal(got, x) and np.array_equal(got.astype(np.float16).astype(float), x)


def test_quantisation_error_is_half_a_step():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((50, 128)) * np.exp2(rng.integers(-8, 8, (50, 1)))).astype(np.float32)
    for fmt, rel, floor in ((od.FP8, 2.0 ** -4, 2.0 ** -10), (od.FP4, 1 / 6, 0.25)):
        codes, scale = od.encode(x, fmt)
        step = np.repeat(2.0 ** (scale.astype(float) - 127), 32, axis=-1)
        err = np.abs(od.decode(codes, scale, fmt) - x)
        assert np.all(err <= np.maximum(rel * np.abs(x), floor * step) * 1.2 + 1e-12)


def test_rotation_is_a_rotation_of_the_pairs():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((3, 2, 64))
    ang = rng.uniform(0, 6, (9, 32))
    y = od.prepare_heads(x, np.array([0, 8, 20]), cos=np.cos(ang), sin=np.sin(ang))
    for t, p in enumerate((0, 8, 8)):
        z = (x[t, :, :32] + 1j * x[t, :, 32:]) * np.exp(1j * ang[p])
        assert np.allclose(y[t], np.concatenate((z.real, z.imag), -1))


def test_attention_against_a_loop_of_sums():
    rng = np.random.default_rng(5)
    q_len, ctx = [3, 1, 2], [5, 4, 1]  # the last sequence's first token has a negative position
    q = rng.standard_normal((6, 4, 8))
    k = [rng.standard_normal((n, 2, 8)) for n in ctx]
    v = [rng.standard_normal((n, 2, 8)) for n in ctx]
    for window in (0, 2):
        out, lse, _ = od.attention(q, k, v, q_len, ctx, 0.3, window)
        t = 0
        for s in range(3):
            for i in range(q_len[s]):
                pos = ctx[s] - q_len[s] + i
                for h in range(4):
                    num, den = np.zeros(8), 0.0
                    for j in range(ctx[s]):
                        if j <= pos and (not window or j > pos - window):
                            w = np.exp(0.3 * float(np.dot(q[t, h], k[s][j, h // 2])))
                            num, den = num + w * v[s][j, h // 2], den + w
                    if den:
                        assert np.allclose(out[t, h], num / den) and np.isclose(lse[t, h], np.log(den))
                    else:
                        assert np.all(out[t, h] == 0) and lse[t, h] == -np.inf
                t += 1
    assert np.all(out[4] == 0) and not np.all(out[5] == 0)


def test_norm_formulas():
    h, y = np.array([[3.0, 4.0]]), np.array([[0.0, 2.0]])
    h2, x = od.norm(h, weight=[1, 2], eps=0.0)
    assert np.allclose(h2, h) and np.allclose(x, [[3 / 12.5 ** .5, 8 / 12.5 ** .5]])
    h2, x = od.norm(h, y=y, post_weight=[1, 1], gate=[5, 0.5], res_scale=2.0, eps=0.0)
    assert x is None and np.allclose(h2, [[3.0, 4.0 + 2 * 0.5 * 2 ** .5]])


def test_pins_reject_planted_mistakes(monkeypatch):
    """A floor for the power of two, ties away from zero, a window one too wide: each fails a pin."""
    real = od._nearest
    monkeypatch.setattr(od, "_nearest", lambda x, m: np.where((lambda i: x == (m[i - 1] + m[i]) / 2)(
        np.clip(np.searchsorted(m, x), 1, len(m) - 1)), np.clip(np.searchsorted(m, x), 1, len(m) - 1), real(x, m)))
    with pytest.raises(AssertionError):
        test_fp4_rounds_to_nearest_ties_to_even()
    monkeypatch.undo()
    real_att = od.attention
    monkeypatch.setattr(od, "attention", lambda q, k, v, a, b, s, w=0: real_att(q, k, v, a, b, s, w + 1 if w else 0))
    with pytest.raises(AssertionError):
        test_attention_against_a_loop_of_sums()
