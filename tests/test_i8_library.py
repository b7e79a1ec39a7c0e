"""Experts in 8-bit integers (HMOE_BF16_I8): the library's host-side quantiser and slot layout against the oracle's, code for
code and scale for scale, and what the host refuses.  No GPU."""
import ctypes

import numpy as np
import pytest

import workloads as wl
from oracle import i8_oracle as i8


@pytest.fixture(scope="module")
def hm():
    import paper_2504_05897_amd as hm
    return hm


def unpack(packed, n_rows, k_len, packed_row):
    """Codes [n_rows, k_len] out of tiles of 32 rows x 32 k: lane l owns row l % 32, k = 16 (l / 32) .. + 16."""
    codes = np.zeros((n_rows, k_len), np.int8)
    for n in range(n_rows):
        pn = packed_row(n)
        for k in range(k_len):
            at = ((pn // 32) * (k_len // 32) + k // 32) * 1024 + (pn % 32 + 32 * (k % 32 // 16)) * 16 + k % 16
            codes[n, k] = packed[at]
    return codes


def test_pack_i8_equals_the_oracle_quantiser(hm):
    hid, ffn = 256, 128
    d = hm.make_desc(hid, ffn, 4, 2, 4, hm.HMOE_BF16_I8)
    n = hid * ffn
    assert hm.hmoe_slot_bytes(d) == 3 * n + 4 * (2 * ffn + hid)
    rng = np.random.default_rng(3)
    mats = [wl.f32_to_bf16_bits((rng.standard_normal(s) * 0.02).astype(np.float32)) for s in ((ffn, hid), (ffn, hid), (hid, ffn))]
    mats[0][5] = 0                                                                        # a row of zeros
    mats[1][9, 4:] = wl.f32_to_bf16_bits(np.linspace(-1, 1, hid - 4, dtype=np.float32))   # many values near halves ...
    mats[1][9, :4] = wl.f32_to_bf16_bits(np.array([254, 1, 3, 127], np.float32))          # ... and some on them: 127 v / 254
    mats[2][7] = wl.f32_to_bf16_bits((rng.standard_normal(ffn) * 1e38).astype(np.float32))   # 127 v is beyond fp32
    mats[2][8] = wl.f32_to_bf16_bits((rng.standard_normal(ffn) * 1e-38).astype(np.float32))  # far below 2^-100
    out = np.zeros(hm.hmoe_slot_bytes(d), np.uint8)
    hm.hmoe_pack_expert(d, *mats, out)
    scales = out[3 * n:].view(np.float32)
    codes = out[:3 * n].view(np.int8)
    for which, (packed, sc, n_rows, k_len, prow) in enumerate([
            (codes[:2 * n], scales[:ffn], ffn, hid, lambda r: 64 * (r // 32) + r % 32),
            (codes[:2 * n], scales[ffn:2 * ffn], ffn, hid, lambda r: 64 * (r // 32) + 32 + r % 32),
            (codes[2 * n:], scales[2 * ffn:], hid, ffn, lambda r: r)]):
        q, s = i8.quantize_rows(wl.as_f64(mats[which]))
        assert np.array_equal(unpack(packed, n_rows, k_len, prow), q), which
        amax = np.maximum(np.abs(wl.as_f32(mats[which])).max(axis=1), np.float32(2.0 ** -100))
        assert np.array_equal(sc, amax / np.float32(127.0)), which
        assert np.allclose(sc, s, rtol=2.0 ** -23, atol=0)


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_pack_i8_marks_rows_that_are_not_finite(hm, value):
    d = hm.make_desc(128, 128, 4, 2, 4, hm.HMOE_BF16_I8)
    w = np.full((128, 128), 0x3f80, np.uint16)
    bad = w.copy()
    bad[3, 5] = np.array([value], np.float32).view(np.uint32)[0] >> 16
    out = np.zeros(hm.hmoe_slot_bytes(d), np.uint8)
    hm.hmoe_pack_expert(d, w, bad, w, out)
    scales = out[3 * 128 * 128:].view(np.float32)
    assert np.isnan(scales[128 + 3]) and np.isfinite(np.delete(scales, 128 + 3)).all()


def test_i8_shape_requirements(hm):
    for hid, ffn in [(192, 128), (128, 192), (64, 64), (131072 + 128, 128), (128, 131072 + 128)]:
        d = hm.make_desc(hid, ffn, 4, 2, 4, hm.HMOE_BF16_I8)
        assert hm.hmoe_slot_bytes(d) == 0
        with pytest.raises(hm.HmoeError) as ei:
            hm.hmoe_pack_expert(d, np.zeros(16, np.uint16), np.zeros(16, np.uint16), np.zeros(16, np.uint16), np.zeros(16, np.uint8))
        assert ei.value.status == hm.HMOE_ERR_UNSUPPORTED
    d = hm.make_desc(256, 384, 4, 2, 4, hm.HMOE_BF16_I8)
    assert hm.hmoe_slot_bytes(d) % 256 == 0
    # h in fp32, the codes of the wider of the two inputs, a scale per row
    assert hm.hmoe_ffn_workspace_bytes(d, 10) >= 10 * (4 * 384 + 384 + 4) and hm.hmoe_ffn_workspace_bytes(d, 0) == 0
    assert hm.hmoe_ffn_workspace_bytes(d, -1) == 0


def test_an_i8_call_is_refused_as_others_are(hm):
    d = hm.make_desc(256, 384, 4, 2, 4, hm.HMOE_BF16_I8)
    lib = hm._lib
    args = [ctypes.byref(d), None, None, None, 4, None, 0, None, None, 0, 0, None]
    assert lib.hmoe_expert_ffn_grouped(*args) == hm.HMOE_ERR_INVALID_ARG                 # no cache
    assert lib.hmoe_pack_expert(ctypes.byref(d), None, None, None, None) == hm.HMOE_ERR_INVALID_ARG


def test_the_oracle_ffn_approaches_the_one_without_codes():
    """Errors of the codes are at most half a step of 1/127 of a row's largest value: the result is near the plain FFN's."""
    from oracle import moe_oracle as orc
    rng = np.random.default_rng(0)
    x, wg, wu, wd = (rng.standard_normal(s) * 0.2 for s in ((5, 256), (128, 256), (128, 256), (256, 128)))
    o, slack = i8.expert_ffn(x, wg, wu, wd)
    ref = orc.expert_ffn(x, wg, wu, wd)
    assert np.abs(o - ref).max() < 0.05 * np.abs(ref).max() and (slack >= 0).all()
