"""4-bit layers and log probabilities without a GPU: sizes, refusals (before any device is touched), and the oracle's layout."""
import numpy as np
import pytest

import paper_2310_19509_b200 as sbnn
from oracle import mxfp4 as O

P = 1 << 20      # an aligned address; no call here gets as far as using it


class T:
    """Something with the address and the type of a tensor."""

    def __init__(self, dtype="float32", at=P, nbytes=1 << 40):
        import torch
        self.dtype, self.at, self.nbytes = getattr(torch, dtype), at, nbytes

    def data_ptr(self):
        return self.at


def name(call, *args, **kw):
    with pytest.raises(sbnn.SbnnError) as e:
        call(*args, stream=0, **kw)
    return e.value.name


def test_bytes():
    assert sbnn.mxfp4_bytes(1, 1) == (16, 512)
    assert sbnn.mxfp4_bytes(0, 7) == (0, 0)
    assert sbnn.mxfp4_bytes(128, 128) == (128 * 64, 512)
    assert sbnn.mxfp4_bytes(129, 129) == (129 * 80, 4 * 512)
    assert sbnn.mxfp4_bytes(2 ** 31 - 1, 2 ** 20)[0] == (2 ** 31 - 1) * 2 ** 19      # past 32 bits
    for m, k in ((-1, 8), (1, 0), (1, -4)):
        with pytest.raises(sbnn.SbnnError) as e:
            sbnn.mxfp4_bytes(m, k)
        assert e.value.name == "SBNN_ERR_SHAPE"


def test_oracle_scale_tiles_are_a_permutation():
    m, k = 300, 517
    off = O.scale_offsets(m, k)
    assert len(np.unique(off)) == off.size and off.max() < sbnn.mxfp4_bytes(m, k)[1]
    b = np.random.default_rng(1).integers(0, 255, (m, O.blocks_of(k))).astype(np.uint8)
    assert np.array_equal(O.tile_scales(b, k)[off], b)


def test_oracle_rounds_ties_to_even_and_saturates():
    x = np.zeros((1, 32))
    x[0, :16] = [.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -7.9]
    c, s = O.quantize(x)
    assert s[0, 0] == 127
    assert np.array_equal(np.abs(O.values(c, s, 32)[0, :8]), [0, 1, 1, 2, 2, 4, 4, 6])


@pytest.mark.parametrize("call", ["quantize", "dequantize"])
def test_quantize_refusals(call):
    fn = sbnn.mxfp4_quantize if call == "quantize" else sbnn.mxfp4_dequantize

    def run(x=T(), ld=64, codes=P, scales=P, m=4, k=64):
        return name(fn, x, ld, codes, scales, m, k) if call == "quantize" else name(fn, codes, scales, x, ld, m, k)

    assert run(x=T(at=0)) == run(codes=None) == run(scales=None) == "SBNN_ERR_NULL"
    assert run(m=-1) == run(k=0) == run(ld=63) == "SBNN_ERR_SHAPE"
    assert run(x=T(at=P + 4)) == run(codes=P + 1) == run(scales=P + 8) == "SBNN_ERR_ALIGN"
    assert run(k=2 ** 30 + 1, ld=2 ** 31) == "SBNN_ERR_UNSUPPORTED"
    with pytest.raises(TypeError):
        run(x=T("float64"))
    fn(*((T(), 64, P, P, 0, 64) if call == "quantize" else (P, P, T(), 64, 0, 64)), stream=0)      # no rows: nothing to do


def test_conv_refusals():
    def run(w=P, ws=P, bias=P, x=T(), ldx=64, y=T(), ldy=48, m=4, cin=64, cout=48, flags=0, work=T("uint8")):
        return name(sbnn.conv1x1_mxfp4, w, ws, bias, x, ldx, y, ldy, m, cin, cout, flags, work)

    assert run(w=None) == run(ws=None) == run(x=T(at=0)) == run(y=T(at=0)) == "SBNN_ERR_NULL"
    assert run(m=-1) == run(cin=0) == run(cout=0) == run(ldx=63) == run(ldy=47) == "SBNN_ERR_SHAPE"
    assert run(flags=sbnn.SBNN_BF16_TC) == "SBNN_ERR_UNSUPPORTED"
    assert run(w=P + 8) == run(ws=P + 4) == run(bias=P + 4) == run(x=T(at=P + 2)) == run(y=T(at=P + 2)) == "SBNN_ERR_ALIGN"
    rows = 33
    need = sum(sbnn.mxfp4_bytes(rows, 64))
    assert run(m=rows, work=None) == "SBNN_ERR_NULL"
    assert run(m=rows, work=T("uint8", nbytes=need - 1)) == "SBNN_ERR_SHAPE"
    assert run(m=rows, work=T("uint8", at=P + 8)) == "SBNN_ERR_ALIGN"
    sbnn.conv1x1_mxfp4(P, P, None, T(), 64, T(), 48, 0, 64, 48, 0, None, stream=0)


def test_conv_q_refusals():
    def run(w=P, ws=P, bias=P, x=P, xs=P, y=T(), ldy=48, m=4, cin=64, cout=48, flags=0):
        return name(sbnn.conv1x1_mxfp4_q, w, ws, bias, x, xs, y, ldy, m, cin, cout, flags)

    assert run(w=None) == run(ws=None) == run(x=None) == run(xs=None) == run(y=T(at=0)) == "SBNN_ERR_NULL"
    assert run(m=-1) == run(cin=0) == run(cout=-3) == run(ldy=47) == "SBNN_ERR_SHAPE"
    assert run(flags=sbnn.SBNN_OUT_CM) == run(m=2 ** 30 + 1) == run(cin=2 ** 30 + 1) == run(cout=2 ** 30 + 1, ldy=2 ** 31) == "SBNN_ERR_UNSUPPORTED"
    assert run(x=P + 8) == run(xs=P + 4) == "SBNN_ERR_ALIGN"


def test_logprobs_refusals():
    def run(x=T(), ld=100, rows=3, classes=100, targets=P, nt=1, lp=P, h=P, top=5, ti=P, tl=P):
        return name(sbnn.logprobs, x, ld, rows, classes, targets, nt, lp, h, top, ti, tl)

    assert run(x=T(at=0)) == run(targets=None) == run(lp=None) == run(ti=None) == run(tl=None) == "SBNN_ERR_NULL"
    assert run(ld=99) == run(rows=-1) == run(classes=0) == run(nt=-1) == "SBNN_ERR_SHAPE"
    assert run(top=-1) == run(top=33) == run(top=11, classes=10, ld=10) == "SBNN_ERR_SHAPE"
    assert run(classes=2 ** 30 + 1, ld=2 ** 31) == "SBNN_ERR_UNSUPPORTED"
    assert run(x=T(at=P + 2)) == run(targets=P + 4) == run(h=P + 8) == "SBNN_ERR_ALIGN"
    sbnn.logprobs(T(), 100, 0, 100, P, 1, P, P, 5, P, P, stream=0)


def test_unknown_element_types_are_refused():
    L = sbnn.lib()
    assert L.sbnn_mxfp4_quantize(P, 3, 64, P, P, 4, 64, None) == 6
    assert L.sbnn_mxfp4_dequantize(P, P, P, -1, 64, 4, 64, None) == 6
    assert L.sbnn_conv1x1_mxfp4(P, P, P, P, 7, 64, P, 0, 64, 4, 64, 64, 0, P, 1 << 40, None) == 6
    assert L.sbnn_conv1x1_mxfp4(P, P, P, P, 0, 64, P, 7, 64, 4, 64, 64, 0, P, 1 << 40, None) == 6
    assert L.sbnn_logprobs(P, 3, 64, 4, 64, P, 1, P, P, 1, P, P, None) == 6
