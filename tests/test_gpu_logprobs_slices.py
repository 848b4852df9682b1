"""Logits that start at any element: rows and columns of a larger tensor."""
import numpy as np
import pytest
import torch

import paper_2310_19509_b200 as sbnn
from oracle import mxfp4 as O
from test_gpu_logprobs import SHAPES, TYPES, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,v", SHAPES + [(40, 1017), (37, 4096), (2, 131072)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("row,column,more", [(1, 0, 1), (0, 1, 0), (0, 3, 5), (2, 7, 1)])
def test_slices(rows, v, dtype, row, column, more):
    """buf[row:, column:column + v]; what lies around would win if it counted.  The same logits in a tensor of their own give the same
    classes, and answers that differ by the order of their sums at most."""
    ld = v + column + more
    x = logits(rows, v, dtype, v + column)
    buf = torch.full((rows + row + 1, ld), 1e4, dtype=x.dtype, device="cuda")
    part = buf[row:row + rows, column:column + v]
    part.copy_(x.cuda())
    t = torch.randint(v, (rows, 2), generator=torch.Generator().manual_seed(v)).int()
    want = O.logprobs(x.double().numpy(), t.numpy(), 6)
    lp, h = torch.empty((rows, 2), device="cuda"), torch.empty((rows,), device="cuda")
    ti, tl = torch.empty((rows, 6), dtype=torch.int32, device="cuda"), torch.empty((rows, 6), device="cuda")
    sbnn.logprobs(part, ld, rows, v, t.cuda(), 2, lp, h, 6, ti, tl)
    sbnn.get_async_status()
    assert np.array_equal(ti.cpu().numpy(), want[2])
    # (shares of at most 1100 terms an accumulator, a few joins: 2^-24 each, and a few steps of values up to 20)
    for got, ref in ((lp, want[0]), (h, want[1]), (tl, want[3])):
        assert np.all(np.abs(got.cpu().double().numpy() - ref) <= 2e-5 + 1e-6 * np.abs(ref))


@pytest.mark.parametrize("dtype", TYPES)
def test_a_start_inside_an_element_is_refused(dtype):
    x = logits(4, 100, dtype).cuda()
    code = {"f32": sbnn.SBNN_F32, "f16": sbnn.SBNN_F16, "bf16": sbnn.SBNN_BF16}[dtype]
    with pytest.raises(sbnn.SbnnError) as e:
        sbnn.logprobs(x.data_ptr() + 1, 100, 3, 100, None, 0, None, None, 0, None, None, logits_type=code)
    assert e.value.name == "SBNN_ERR_ALIGN"
