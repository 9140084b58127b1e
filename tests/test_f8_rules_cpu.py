"""Refusals and size queries of the 8-bit product and of the rules on logits: all checks come before any device call, so they
run without a GPU."""

import ctypes

import pytest

from paper_1805_11462_amd import _lib
from paper_1805_11462_amd._lib import OnmtLogitRules

P = 1 << 20            # an aligned address that is never read
WS, OUT, W = 1 << 30, 1 << 34, 1 << 40


def test_sizes():
    lib = _lib.load()
    # 2 KB per 16 x 128 block, 64 bytes per 16 rows and four blocks
    assert lib.onmt_f8_bytes(1, 1) == 2048 + 64
    assert lib.onmt_f8_bytes(17, 129) == 4 * 2048 + 2 * 64
    assert lib.onmt_f8_bytes(50000, 500) == 3125 * (4 * 2048 + 64)
    assert lib.onmt_f8_bytes(16, 513) == 5 * 2048 + 2 * 64
    for bad in ((0, 4), (4, 0), (-1, 4), (1 << 30, 1 << 10)):
        assert lib.onmt_f8_bytes(*bad) == 0
        assert lib.onmt_f8_linear_ws_bytes(*bad) == 0
    assert lib.onmt_f8_linear_ws_bytes(100, 500) >= 100 * 500
    assert lib.onmt_constrain_ws_bytes(4, 1000, 2, 0) == 0
    assert lib.onmt_constrain_ws_bytes(4, 1000, 0, 0) > 0
    assert lib.onmt_constrain_ws_bytes(4, 1000, 1, 17) == 0
    assert lib.onmt_constrain_ws_bytes(4, (1 << 20) + 1, 0, 1) == 0


def linear(**kw):
    a = dict(x=P, dtype=0, ldx=500, M=5, packed=W, pbytes=1 << 39, rows=1000, cols=500, bias=None, out=OUT, out_dtype=0,
             ld_out=1000, ws=WS, ws_bytes=1 << 30)
    assert set(kw) <= set(a)
    a.update(kw)
    return _lib.load().onmt_f8_linear(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), _lib.ONMT_EINVAL), (dict(x=P + 2), _lib.ONMT_EINVAL), (dict(x=P + 1, dtype=1), _lib.ONMT_EINVAL),
    (dict(dtype=3), _lib.ONMT_EINVAL), (dict(out_dtype=-1), _lib.ONMT_EINVAL), (dict(ldx=499), _lib.ONMT_EINVAL),
    (dict(ldx=-500), _lib.ONMT_EINVAL), (dict(ldx=1 << 62), _lib.ONMT_EINVAL), (dict(M=0), _lib.ONMT_EINVAL),
    (dict(packed=None), _lib.ONMT_EINVAL), (dict(packed=W + 8), _lib.ONMT_EINVAL), (dict(pbytes=63 * 4 * 2048), _lib.ONMT_ESIZE),
    (dict(rows=0), _lib.ONMT_EINVAL), (dict(out=None), _lib.ONMT_EINVAL), (dict(ld_out=999), _lib.ONMT_EINVAL),
    (dict(bias=P + 1), _lib.ONMT_EINVAL), (dict(M=100, ws=None), _lib.ONMT_EINVAL), (dict(M=100, ws=WS + 4), _lib.ONMT_EINVAL),
    (dict(M=100, ws_bytes=64), _lib.ONMT_ESIZE),
    # out over x, over the workspace, over the weights
    (dict(out=P), _lib.ONMT_EINVAL), (dict(out=P + 5 * 500 * 4 - 4), _lib.ONMT_EINVAL), (dict(M=100, out=WS), _lib.ONMT_EINVAL),
    (dict(out=W + 64), _lib.ONMT_EINVAL), (dict(bias=OUT + 4 * 4999), _lib.ONMT_EINVAL),
    # the workspace over x, over the weights, over the bias
    (dict(M=100, ws=P), _lib.ONMT_EINVAL), (dict(M=100, ws=W), _lib.ONMT_EINVAL), (dict(M=100, bias=WS), _lib.ONMT_EINVAL),
    (dict(M=1 << 30, ldx=500), _lib.ONMT_EUNSUPPORTED),
])
def test_linear_refusals(kw, code):
    assert linear(**kw) == code
    assert len(_lib.load().onmt_last_error()) > 0


def test_generator_needs_a_model():
    assert _lib.load().onmt_set_generator(None, P, 1 << 30) == _lib.ONMT_EINVAL
    assert _lib.load().onmt_set_generator(None, None, 0) == _lib.ONMT_EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(w=None), _lib.ONMT_EINVAL), (dict(dtype=9), _lib.ONMT_EINVAL), (dict(ld=3), _lib.ONMT_EINVAL),
    (dict(nbytes=100), _lib.ONMT_ESIZE), (dict(packed=None), _lib.ONMT_EINVAL), (dict(rows=1 << 28, nbytes=1 << 62), _lib.ONMT_EUNSUPPORTED),
])
def test_pack_refusals(kw, code):
    a = dict(w=P, dtype=0, ld=128, rows=16, cols=128, packed=W, nbytes=1 << 30)
    a.update(kw)
    if "rows" in kw:
        a["cols"], a["ld"] = 1 << 12, 1 << 12
    assert _lib.load().onmt_f8_pack(*a.values(), None) == code
    if "w" not in kw and "dtype" not in kw:
        assert _lib.load().onmt_f8_unpack(a["packed"], a["nbytes"], a["rows"], a["cols"], P, a["ld"], None) == code


def constrain(rules=None, **kw):
    a = dict(logits=P, dtype=0, ld=1000, N=4, V=1000, mode=1, K=5, out=OUT, ld_out=5, ids=W, lse=None, ws=WS,
             ws_bytes=1 << 30)
    assert set(kw) <= set(a)
    a.update(kw)
    ref = None
    if rules is not None:
        ref = ctypes.byref(OnmtLogitRules(**rules))
    return _lib.load().onmt_constrain(ref, *a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), _lib.ONMT_EINVAL), (dict(dtype=4), _lib.ONMT_EINVAL), (dict(ld=999), _lib.ONMT_EINVAL),
    (dict(N=0), _lib.ONMT_EINVAL), (dict(V=0), _lib.ONMT_EINVAL), (dict(mode=3), _lib.ONMT_EINVAL),
    (dict(mode=-1), _lib.ONMT_EINVAL), (dict(K=0), _lib.ONMT_EUNSUPPORTED), (dict(K=17, ld_out=17), _lib.ONMT_EUNSUPPORTED),
    (dict(V=4, ld=4), _lib.ONMT_EINVAL), (dict(ids=None), _lib.ONMT_EINVAL), (dict(ids=W + 1), _lib.ONMT_EINVAL),
    (dict(ld_out=6), _lib.ONMT_EINVAL), (dict(out=None), _lib.ONMT_EINVAL), (dict(ws=None), _lib.ONMT_EINVAL),
    (dict(ws_bytes=8), _lib.ONMT_ESIZE), (dict(out=P), _lib.ONMT_EINVAL), (dict(out=WS), _lib.ONMT_EINVAL),
    (dict(ws=P), _lib.ONMT_EINVAL),
    (dict(mode=2, ld_out=1000, lse=W), _lib.ONMT_EINVAL),
    # in place needs the same pointer, stride and type
    (dict(mode=2, out=P + 4, ld_out=1000), _lib.ONMT_EINVAL), (dict(mode=2, out=P, ld_out=1001), _lib.ONMT_EINVAL),
    (dict(mode=0, dtype=1, out=P, ld_out=1000), _lib.ONMT_EINVAL),
    (dict(V=(1 << 20) + 1, ld=1 << 21), _lib.ONMT_EUNSUPPORTED), (dict(N=1 << 24), _lib.ONMT_EUNSUPPORTED),
])
def test_constrain_refusals(kw, code):
    assert constrain(**kw) == code
    assert len(_lib.load().onmt_last_error()) > 0


@pytest.mark.parametrize("rules", [
    dict(history=P, history_stride=10, max_history=10),                                  # no lengths
    dict(history=P, history_len=P, history_stride=9, max_history=10),
    dict(history=P, history_len=P, history_stride=9, max_history=0),
    dict(history=P + 2, history_len=P, history_stride=10, max_history=10),
    dict(no_repeat_ngram=-1),
    dict(n_bias=-1), dict(n_bias=3, bias_ids=P, bias_stride=3), dict(n_bias=3, bias_ids=P, bias=P, bias_stride=2),
    dict(history=P, history_len=P, history_stride=1 << 20, max_history=65536), dict(n_bias=65536, bias_ids=P, bias=P, bias_stride=65536),
    dict(mask=P, mask_stride=31, n_masks=4), dict(mask=P, mask_stride=32, n_masks=0, mask_row=P),
    dict(mask=P, mask_stride=32, n_masks=3),                                             # a table per row: four are needed
    dict(mask=P, mask_stride=32, n_masks=1, mask_row=P + 1),
])
def test_rules_refusals(rules):
    long = rules.get("max_history", 0) > 65535 or rules.get("n_bias", 0) > 65535
    assert constrain(rules) == (_lib.ONMT_EUNSUPPORTED if long else _lib.ONMT_EINVAL)
    assert len(_lib.load().onmt_last_error()) > 0
