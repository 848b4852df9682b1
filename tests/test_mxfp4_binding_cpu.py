"""Addresses and None in the place of tensors, as every entry point of the binding takes them.  No GPU."""
import pytest

import paper_2310_19509_b200 as sbnn
from test_mxfp4_cpu import P, T, name

F16 = sbnn.SBNN_F16


def test_none_is_refused_by_the_library():
    assert name(sbnn.mxfp4_quantize, None, 64, P, P, 4, 64) == "SBNN_ERR_NULL"
    assert name(sbnn.mxfp4_dequantize, P, P, None, 64, 4, 64) == "SBNN_ERR_NULL"
    assert name(sbnn.conv1x1_mxfp4, P, P, None, None, 64, T(), 48, 4, 64, 48, 0) == "SBNN_ERR_NULL"
    assert name(sbnn.conv1x1_mxfp4, P, P, None, T(), 64, None, 48, 4, 64, 48, 0) == "SBNN_ERR_NULL"
    assert name(sbnn.conv1x1_mxfp4_q, P, P, None, P, P, None, 48, 4, 64, 48, 0) == "SBNN_ERR_NULL"
    assert name(sbnn.logprobs, None, 9, 4, 9, None, 0, None, None, 0, None, None) == "SBNN_ERR_NULL"


def test_addresses_with_their_types():
    """No rows: accepted; addresses that the library refuses: they got there."""
    sbnn.mxfp4_quantize(P, 64, P, P, 0, 64, stream=0, x_type=F16)
    sbnn.mxfp4_dequantize(P, P, P, 64, 0, 64, stream=0, y_type=F16)
    sbnn.conv1x1_mxfp4(P, P, None, P, 64, P, 48, 0, 64, 48, 0, P, stream=0, x_type=F16, y_type=sbnn.SBNN_BF16, workspace_bytes=1 << 20)
    sbnn.conv1x1_mxfp4_q(P, P, None, P, P, P, 48, 0, 64, 48, 0, stream=0, y_type=F16)
    sbnn.logprobs(P, 9, 0, 9, None, 0, None, None, 0, None, None, stream=0, logits_type=F16)
    assert name(sbnn.mxfp4_quantize, P + 2, 64, P, P, 4, 64, x_type=F16) == "SBNN_ERR_ALIGN"
    assert name(sbnn.conv1x1_mxfp4, P, P, None, P, 64, P, 48, 64, 64, 48, 0, P, x_type=F16, y_type=F16, workspace_bytes=5) == "SBNN_ERR_SHAPE"
    assert name(sbnn.mxfp4_quantize, P, 64, P, P, 4, 64, x_type=3) == "SBNN_ERR_UNSUPPORTED"


def test_an_address_without_a_type_is_a_type_error():
    for call in (lambda: sbnn.mxfp4_quantize(P, 64, P, P, 4, 64, stream=0), lambda: sbnn.mxfp4_dequantize(P, P, P, 64, 4, 64, stream=0),
                 lambda: sbnn.logprobs(P, 9, 4, 9, None, 0, None, None, 0, None, None, stream=0)):
        with pytest.raises(TypeError):
            call()


def test_logits_start_at_any_element():
    for dtype, size in (("float32", 4), ("float16", 2), ("bfloat16", 2)):
        sbnn.logprobs(T(dtype, at=P + size), 9, 0, 9, None, 0, None, None, 0, None, None, stream=0)
        assert name(sbnn.logprobs, T(dtype, at=P + size // 2), 9, 4, 9, None, 0, None, None, 0, None, None) == "SBNN_ERR_ALIGN"
