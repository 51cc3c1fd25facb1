"""The serving oracle pinned on what is known in closed form (CPU)."""
import numpy as np

from oracle import attend_oracle as orc


def test_e4m3_table():
    v = orc.e4m3_values()
    assert v[0x7E] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1.0 and v[0xB8] == -1.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and np.all(np.diff(v[:127]) > 0)


def test_codes_of_representable_rows_are_exact():
    v = orc.e4m3_values()[:127]
    for e in (-20, 0, 13):
        code, exp = orc.quantize_rows(v * 2.0 ** e)
        assert exp == e + 127 and np.array_equal(code, np.arange(127))
        assert np.array_equal(orc.dequantize_rows(code, exp), v * 2.0 ** e)


def test_scale_is_the_smallest_that_fits():
    x = np.zeros((4, 8))
    x[:, 0] = 448.0, 448.0001, 1e-300, 0.0
    code, exp = orc.quantize_rows(x)
    assert exp.tolist() == [127, 128, 0, 0] and code[0, 0] == 0x7E and code[3, 0] == 0


def test_ties_go_to_even_and_nonfinite_to_nan():
    code, exp = orc.quantize_rows(np.array([448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, np.inf, np.nan, -np.inf]))
    val = orc.dequantize_rows(code, exp)
    assert exp == 127 and val[1] == 16.0 and val[2] == 20.0 and val[3] == 0.0 and val[4] == 2.0 ** -8
    assert np.isnan(val[5:]).all()


def test_attention_of_equal_keys_is_the_mean():
    v = np.arange(12.0).reshape(4, 3)
    out, lse, absv, _ = orc.attend_row(np.ones(3), np.zeros((4, 3)), v, 0.7)
    assert np.allclose(out, v.mean(0)) and np.isclose(lse, np.log(4)) and np.allclose(absv, out)
    out, lse, _, _ = orc.attend_row(np.ones(3), np.zeros((0, 3)), np.zeros((0, 3)), 0.7)
    assert np.all(out == 0) and lse == -np.inf


def test_attention_follows_a_dominant_key():
    k = np.zeros((5, 2))
    k[3, 0] = 100.0
    v = np.eye(5)
    out, lse, _, _ = orc.attend_row(np.array([2.0, 0.0]), k, v, 1.0)
    assert np.allclose(out, v[3]) and np.isclose(lse, 200.0)


def test_largest_bf16_stays_finite():
    code, exp = orc.quantize_rows(np.array([2.0 ** 128 * (1 - 2.0 ** -8), -3.3e38, 1.0]))
    assert exp == 247 and np.array_equal(orc.dequantize_rows(code, exp)[:2], [240 * 2.0 ** 120, -240 * 2.0 ** 120])
