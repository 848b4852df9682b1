"""Every form that a 4-bit layer runs in, with every output type, ReLU, strides, both entries, and guards around what is written."""
import functools

import numpy as np
import pytest
import torch

import paper_2310_19509_b200 as sbnn
from oracle import mxfp4 as O
from test_gpu_mxfp4 import TYPES, activations, bound

pytestmark = pytest.mark.gpu
CODE = {"f32": sbnn.SBNN_F32, "f16": sbnn.SBNN_F16, "bf16": sbnn.SBNN_BF16}

# (m, k, n) -> pairs of CTAs, pixels of a tile, CTAs that share it.  Pixels, channels and output channels fill no tile.
# A third entry: what half-precision outputs run on, where that differs (pairs write those in less time).
FORMS = {
    "pairs": ((1301, 517, 4088), (True, 256, 1)),
    "pairs, rows that the copy engine cannot write": ((1301, 517, 4090), (True, 256, 1)),
    "pairs, more steps than stages": ((300, 4096, 4099), (True, 256, 1)),
    "pairs, one block": ((519, 8, 3717), (True, 256, 1)),
    "tiles of 256": ((1078, 40, 3669), (False, 256, 1)),
    "tiles of 256, more steps than stages": ((575, 1088, 6187), (False, 256, 1), (True, 256, 1)),
    "tiles of 128": ((3223, 40, 260), (False, 128, 1)),
    "tiles of 128 shared": ((600, 4096, 1000), (False, 128, 3)),
    "tiles of 64": ((196, 517, 516), (False, 64, 1)),
    "tiles of 64 shared by 3": ((1668, 1419, 8), (False, 64, 3)),
    "tiles of 64 shared by 8": ((37, 1803, 9), (False, 64, 8)),
    "few pixels": ((13, 517, 300), (False, 16, 1)),
    "few pixels, shared": ((27, 2050, 300), (False, 32, 5)),
}


def plan(m, k, n, dtype, pre):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    return sbnn.debug_plan_conv1x1_mxfp4(m, k, n, CODE[dtype], 0 if pre else 2, sms)[:3]


class Weights:
    """Codes and scales that are drawn as such; rows of no channel have the scale 255, which must not matter."""

    def __init__(self, n, k, seed):
        rng = np.random.default_rng(seed)
        codes = rng.integers(0, 256, (n, 16 * O.blocks_of(k))).astype(np.uint8)
        if k % 32:                                    # elements behind the last channel are 0
            last = codes[:, -16:]
            lo, hi = last & 15, last >> 4
            at = np.arange(16)
            codes[:, -16:] = np.where(2 * at < k % 32, lo, 0) | np.where(2 * at + 1 < k % 32, hi, 0) << 4
        scales = rng.integers(118, 124, (n, O.blocks_of(k))).astype(np.uint8)
        self.values = O.values(codes, scales, k)
        self.codes, self.scales = torch.from_numpy(codes).cuda(), torch.from_numpy(O.tile_scales(scales, k, 255)).cuda()
        self.bias = rng.standard_normal(n).astype(np.float32) * 4
        self.bias_dev = torch.from_numpy(self.bias).cuda()


@functools.lru_cache(maxsize=1)
def layer_of(form):
    """(weights, activations, their 4-bit form, sums in 64 bits, what errors are measured by)."""
    m, k, n = FORMS[form][0]
    w, x = Weights(n, k, m), activations(m, k, "f32", n)
    xc, xs = O.quantize(x.double().numpy())
    y, s = O.conv1x1(O.values(xc, xs, k), w.values, w.bias, False)
    return w, x, xc, xs, y, s


def call(w, x, xc, xs, m, k, n, dtype, relu=False, pre=False, ldx=None, ldy=None, bias=True, out=None):
    """Runs the layer; returns its outputs [m][n] after looking at everything around them.  `out`: (whole, offset) to write to again."""
    ldx, ldy = ldx or k, ldy or n
    front, back = 1024, 1024 + ldy
    whole = torch.full((front + m * ldy + back,), 7.0, dtype=TYPES[dtype], device="cuda")
    y = whole[front:front + m * ldy].view(m, ldy)
    flags = sbnn.SBNN_RELU if relu else 0
    b = w.bias_dev if bias else None
    if pre:
        sbnn.conv1x1_mxfp4_q(w.codes, w.scales, b, torch.from_numpy(xc).cuda(), torch.from_numpy(O.tile_scales(xs, k, 255)).cuda(), y, ldy, m, k, n, flags)
    else:
        xd = torch.full((m, ldx), float("nan"), device="cuda")
        xd[:, :k] = x.cuda()
        need = sum(sbnn.mxfp4_bytes(m, k))
        work = torch.full((need + 1024,), 0xA5, dtype=torch.uint8, device="cuda")
        sbnn.conv1x1_mxfp4(w.codes, w.scales, b, xd, ldx, y, ldy, m, k, n, flags, work[512:512 + need])
        assert bool((work[:512] == 0xA5).all()) and bool((work[512 + need:] == 0xA5).all()), "written outside the workspace"
    sbnn.get_async_status()
    assert bool((whole[:front] == 7.0).all()), "written in front of the outputs"
    assert bool((whole[front + m * ldy:] == 7.0).all()), "written behind the outputs"
    assert bool((y[:, n:] == 7.0).all()), "written between the rows"
    return y[:, :n]


def check(got, ref, s, k, dtype):
    worst = np.abs(got.cpu().double().numpy() - ref) / bound(k, s, ref, dtype)
    assert np.all(worst <= 1), f"worst {np.nanmax(worst)} of the bound"


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_forms(form, dtype, relu, pre):
    (m, k, n), *expected = FORMS[form]
    assert plan(m, k, n, dtype, pre) == expected[0 if dtype == "f32" else -1]
    w, x, xc, xs, ref, s = layer_of(form)
    check(call(w, x, xc, xs, m, k, n, dtype, relu, pre), np.maximum(ref, 0) if relu else ref, s, k, dtype)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("more", [(8, 8), (3, 1), (0, 5), (1, 264)])
def test_strides(form, dtype, more):
    m, k, n = FORMS[form][0]
    w, x, xc, xs, ref, s = layer_of(form)
    check(call(w, x, xc, xs, m, k, n, dtype, ldx=k + more[0], ldy=n + more[1]), ref, s, k, dtype)


@pytest.mark.parametrize("form", FORMS)
def test_no_bias(form):
    m, k, n = FORMS[form][0]
    w, x, xc, xs, ref, s = layer_of(form)
    check(call(w, x, xc, xs, m, k, n, "bf16", bias=False), ref - w.bias.astype(np.float64), s, k, "bf16")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("pre", [False, True])
@pytest.mark.parametrize("relu", [False, True])
def test_bad_and_empty_blocks(form, pre, relu):
    """NaN and infinities in one block of the first, a middle and the last pixel reach all outputs of those and no other; blocks, pixels
    and channels of zeros between them."""
    m, k, n = FORMS[form][0]
    w, x, _, _, _, _ = layer_of(form)
    x = x.clone()
    x[:, k // 2:k // 2 + 40] = 0
    x[m // 3] = 0
    bad = sorted({0, m // 2, m - 1})
    for r, v in zip(bad, (float("nan"), float("inf"), -float("inf"))):
        x[r, (r * 7) % k] = v
    xc, xs = O.quantize(x.double().numpy())
    xv = O.values(xc, xs, k)
    got = call(w, x, xc, xs, m, k, n, "f32", relu, pre)
    xv[bad] = 0
    ref, s = O.conv1x1(xv, w.values, w.bias, relu)
    lost = got[torch.tensor(bad, device="cuda")].cpu()
    assert bool((lost == 0).all()) if relu else bool(lost.isnan().all())     # max(NaN, 0) is 0
    keep = np.setdiff1d(np.arange(m), bad)
    check(got[torch.from_numpy(keep).cuda()], ref[keep], s[keep], k, "f32")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_entries_repeats_and_replays_agree(form, dtype):
    """Both entries, calls again and replays of a captured call, all behind each other in a stream, give the same bits."""
    m, k, n = FORMS[form][0]
    w, x, xc, xs, _, _ = layer_of(form)
    want = call(w, x, xc, xs, m, k, n, dtype)
    for pre in (True, False):
        assert torch.equal(call(w, x, xc, xs, m, k, n, dtype, pre=pre), want)
    xd, xn = x.cuda(), torch.zeros_like(x, device="cuda")
    work = torch.empty((sum(sbnn.mxfp4_bytes(m, k)),), dtype=torch.uint8, device="cuda")
    y = [torch.zeros((m, n), dtype=TYPES[dtype], device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(3):                            # one workspace, one after the other
            sbnn.conv1x1_mxfp4(w.codes, w.scales, w.bias_dev, xn, k, y[i], n, m, k, n, 0, work)
    for _ in range(3):
        xn.copy_(xd)
        graph.replay()
        xn.zero_()
        for v in y:
            assert torch.equal(v, want)
            v.zero_()
    sbnn.get_async_status()


@pytest.mark.parametrize("form", ["pairs", "tiles of 256", "tiles of 64 shared by 3", "few pixels, shared"])
def test_two_streams_at_once(form):
    """Calls on two streams that share weights and nothing else."""
    m, k, n = FORMS[form][0]
    w, x, xc, xs, _, _ = layer_of(form)
    want = call(w, x, xc, xs, m, k, n, "bf16").clone()
    xd = x.cuda()
    streams = [torch.cuda.Stream() for _ in range(2)]
    y = [[torch.zeros((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(6)] for _ in streams]
    work = [torch.empty((sum(sbnn.mxfp4_bytes(m, k)),), dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    for i in range(6):
        for j, st in enumerate(streams):
            sbnn.conv1x1_mxfp4(w.codes, w.scales, w.bias_dev, xd, k, y[j][i], n, m, k, n, 0, work[j], stream=st)
    torch.cuda.synchronize()
    sbnn.get_async_status()
    assert all(torch.equal(v, want) for side in y for v in side)


@pytest.mark.parametrize("form", FORMS)
def test_bad_weights_reach_their_channel_and_no_other(form):
    """Blocks of NaN in the first, a middle and the last output channel."""
    m, k, n = FORMS[form][0]
    w, x, xc, xs, ref, s = layer_of(form)
    want = call(w, x, xc, xs, m, k, n, "f32")
    bad = sorted({0, n // 2, n - 1})
    kept = w.scales
    w.scales = kept.clone()
    off = O.scale_offsets(n, k)
    for r, b in zip(bad, (0, off.shape[1] - 1, off.shape[1] // 2)):
        w.scales[int(off[r, b])] = 255
    try:
        got = call(w, x, xc, xs, m, k, n, "f32")
    finally:
        w.scales = kept
    at = torch.tensor(bad, device="cuda")
    assert bool(got[:, at].isnan().all())
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[at] = False
    assert torch.equal(got[:, keep], want[:, keep])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("ex", [-118, -90, 90, 110])
def test_scales_of_opposite_ends(form, ex):
    """Activations times 2^ex and weights over 2^ex: the same products, whose scales lie near the ends of their range, and so the same bits."""
    m, k, n = FORMS[form][0]
    w, x, xc, xs, ref, s = layer_of(form)
    want = call(w, x, xc, xs, m, k, n, "f32")
    kept = w.scales
    there = (kept != 255) & (kept != 0)               # rows of no channel and blocks behind the last keep their bytes
    w.scales = torch.where(there, (kept.int() - ex).clamp(0, 254).to(torch.uint8), kept)
    moved = np.where(xs > 0, xs.astype(np.int64) + ex, 0)
    assert moved.max() <= 254 and moved[xs > 0].min() >= 0 and int(kept[there].min()) - ex >= 0
    try:
        got = call(w, x, xc, moved.astype(np.uint8), m, k, n, "f32", pre=True)
    finally:
        w.scales = kept
    assert torch.equal(got, want)
