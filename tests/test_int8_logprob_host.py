"""Without a GPU: the oracles of 8-bit products and log-probabilities against closed forms, and the refusals of their entry points."""
import ctypes as C

import numpy as np
import pytest

from oracle import int8_oracle as Q
from oracle import logprob_oracle as L
from paper_2506_10470_amd import tdp


def test_quantisation_by_hand():
    codes, scales = Q.quantise(np.array([[127, -64, 0.5, 1.5], [0, 0, 0, 0], [1, np.nan, 2, 3], [-np.inf, 1, 1, 1], [2.0 ** -132, -2.0 ** -133, 0, 0]],
                                        dtype=np.float32))
    assert codes[0].tolist() == [127, -64, 0, 2] and scales[0] == 1     # ties to the even code
    assert (codes[1] == 0).all() and scales[1] == 0
    assert (codes[2:4] == 0).all() and np.isnan(scales[2:4]).all()
    assert codes[4].tolist() == [127, -64, 0, 0] and 0 < scales[4] < 1e-41   # -63.5: the even of -64 and -63


def test_quantised_values_are_within_half_a_scale():
    v = np.random.default_rng(2).standard_normal((50, 333)).astype(np.float32)
    codes, scales = Q.quantise(v)
    assert np.abs(codes).max(1).tolist() == [127] * 50
    assert (np.abs(codes * scales[:, None].astype(np.float64) - v) <= scales[:, None] * (0.5 + 1e-4)).all()


def test_quantised_values_of_every_magnitude_are_within_the_stated_distance():
    """(1/2 + 2^-15) scales, 381 roundings of 2^-24 beside the half; 2^-143 more, 127 codes of half of 2^-149, where the scale is subnormal."""
    rng = np.random.default_rng(4)
    with np.errstate(under="ignore"):
        v = (rng.uniform(-1, 1, (3000, 40)) * 2.0 ** rng.uniform(-149, 127, (3000, 1))).astype(np.float32)
    codes, scales = Q.quantise(v)
    scales = scales.astype(np.float64)[:, None]
    off = np.abs(codes * scales - v.astype(np.float64))
    subnormal = scales < 2.0 ** -126
    assert subnormal.any() and (scales == 0).any() and np.abs(codes).max() == 127
    assert (off <= scales * (0.5 + 2.0 ** -15) + np.where(subnormal, 2.0 ** -143, 0)).all()


def test_product_by_hand():
    y = Q.product(np.array([[1, 2], [3, -4]]), [0.5, 2], np.array([[10, 20], [-1, 0], [0, 1]]), [1, 4, 0.25])
    assert y.tolist() == [[25, -2, 0.25], [-100, -24, -2]]


def test_log_probabilities_by_hand():
    z = np.array([[0.0, np.log(2), np.log(5)], [3, 3, 3], [-np.inf, 0, -np.inf], [-np.inf] * 3, [np.nan, 1, 2], [np.inf, 0, 0]])
    lp, en, ix, tl = L.answer(z, [1, -1, 0, 1, 3, 1], 2)
    assert np.allclose(lp[:3], [np.log(0.25), -np.inf, -np.inf]) and np.isnan(lp[3]) and lp[4] == -np.inf and np.isnan(lp[5])
    p = np.array([1, 2, 5]) / 8
    assert np.allclose(en[:3], [-(p * np.log(p)).sum(), np.log(3), 0]) and np.isnan(en[3:]).all()
    assert ix.tolist() == [[2, 1], [0, 1], [1, 0], [0, 1], [2, 1], [0, 1]]
    assert np.allclose(tl[0], np.log([5 / 8, 2 / 8])) and np.isnan(tl[3:]).all()


def test_the_greedy_log_probability_is_that_of_the_largest_logit():
    z = np.random.default_rng(3).standard_normal((4, 30))
    lp, _, ix, tl = L.answer(z, None, 1)
    assert np.array_equal(lp, tl[:, 0]) and np.array_equal(ix[:, 0], z.argmax(1))


@pytest.mark.parametrize("bad", [dict(in_features=0), dict(in_features=12), dict(in_features=131080), dict(out_features=0), dict(out_features=6),
                                 dict(out_features=4, gated=1), dict(gated=2), dict(max_rows=0), dict(max_rows=-1), dict(out_features=1 << 25)])
def test_products_in_8_bits_reject_bad_configurations(bad):
    cfg = dict(in_features=64, out_features=64, gated=0, max_rows=4)
    cfg.update(bad)
    with pytest.raises(tdp.TdpError) as e:
        tdp.tdp_linear_i8_create(tdp.LinearI8Config(**cfg))
    assert e.value.code == tdp.EINVAL and tdp.last_error()


def test_products_in_8_bits_reject_null_arguments():
    h = C.c_void_p()
    assert tdp.lib.tdp_linear_i8_create(None, C.byref(h)) == tdp.EINVAL
    assert tdp.lib.tdp_linear_i8_set_weight(None, 16, 0, 0, 8, 4) == tdp.EINVAL
    assert tdp.lib.tdp_linear_i8_set_codes(None, 16, 16, 0, 8, 4) == tdp.EINVAL
    assert tdp.lib.tdp_linear_i8_set_bias(None, 16, 0, 0, 4) == tdp.EINVAL
    assert tdp.lib.tdp_linear_i8_set_form(None, 0, 1) == tdp.EINVAL
    assert tdp.lib.tdp_linear_i8_run(None, 16, 1, 8, 1, None, 0, 16, 1, 4, None) == tdp.EINVAL
    tdp.lib.tdp_linear_i8_destroy(None)


def test_log_probabilities_reject_bad_arguments():
    R = tdp.lib.tdp_logprob_rows
    for dtype, M, n, ld, n_top in [(2, 1, 8, 8, 0), (-1, 1, 8, 8, 0), (0, -1, 8, 8, 0), (0, 1, 0, 8, 0), (0, 1, 8, 7, 0), (0, 1, 8, 8, -1),
                                   (0, 1, 8, 8, 9), (0, 1, 100, 100, 33), (0, 1, (1 << 30) + 1, 1 << 31, 0)]:
        assert R(4096, dtype, M, n, ld, None, n_top, None, None, 4096, 4096, None) == tdp.EINVAL, (dtype, M, n, ld, n_top)
    assert R(None, 0, 1, 8, 8, None, 0, None, None, None, None, None) == tdp.EINVAL          # no logits
    assert R(4096, 0, 1, 8, 8, None, 2, None, None, None, 4096, None) == tdp.EINVAL          # tokens wanted, nowhere to put them
    assert R(4096, 0, 1, 8, 8, None, 2, None, None, 4096, None, None) == tdp.EINVAL
    assert R(4098, 0, 1, 8, 8, None, 0, None, None, None, None, None) == tdp.EINVAL          # fp32 at an odd address
    assert R(4097, 1, 1, 8, 8, None, 0, None, None, None, None, None) == tdp.EINVAL
    assert R(None, 0, 0, 8, 8, None, 0, None, None, None, None, None) == tdp.OK              # empty is a no-op
    assert tdp.lib.tdp_lm_head_logprobs(None, None, 1, None, 1, None, 0, None, None, None, None, None, None) == tdp.EINVAL
