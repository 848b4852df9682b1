"""4-bit quantisation and the 1x1 layer on 4-bit operands against their definition in 64 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2310_19509_b200 as sbnn
from oracle import mxfp4 as O

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
GUARD = 0xA5
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def guarded(nbytes, fill=GUARD):
    """A uint8 buffer with 512 guard bytes on either side; (whole, the part between)."""
    whole = torch.full((nbytes + 1024,), fill, dtype=torch.uint8, device="cuda")
    return whole, whole[512:512 + nbytes]


def intact(whole):
    assert bool((whole[:512] == GUARD).all()) and bool((whole[-512:] == GUARD).all()), "written outside"


def activations(m, k, dtype, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((m, k), generator=g) * torch.exp(spread * torch.randn((k,), generator=g))
    return x.to(TYPES[dtype])


def strided(x, ld):
    """The rows of x on the device, ld elements apart, the gaps full of NaN."""
    m, k = x.shape
    buf = torch.full((m, ld), float("nan"), dtype=x.dtype, device="cuda")
    buf[:, :k] = x.cuda()
    return buf


def quantized(x, ld=None):
    """Codes and scales of the device's quantisation, checked for what it must leave alone."""
    m, k = x.shape
    cb, sb = sbnn.mxfp4_bytes(m, k)
    wc, codes = guarded(cb)
    ws, scales = guarded(sb)
    xd = strided(x, ld or k)
    sbnn.mxfp4_quantize(xd, ld or k, codes, scales, m, k)
    sbnn.get_async_status()
    intact(wc), intact(ws)
    return codes, scales


def check_quantize(x, ld=None):
    m, k = x.shape
    codes, scales = quantized(x, ld)
    want_c, want_s = O.quantize(x.double().numpy())
    assert np.array_equal(codes.cpu().numpy().reshape(m, -1), want_c)
    # rows behind m keep what was there
    assert np.array_equal(scales.cpu().numpy(), O.tile_scales(want_s, k, GUARD))
    return codes, scales, want_c, want_s


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k", [(1, 1), (1, 31), (1, 32), (2, 33), (1, 1024), (5, 129), (33, 96), (127, 128), (128, 160), (129, 517), (300, 256), (257, 1000),
                                 (40000, 40), (38000, 64), (39000, 100), (37890, 128), (9000, 1001), (4800, 2048)])
def test_quantize_is_exact(m, k, dtype):
    check_quantize(activations(m, k, dtype, 7 * m + k))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ld", [517, 520, 523, 1024])
def test_quantize_strides(ld, dtype):
    check_quantize(activations(130, 517, dtype, 3), ld)
    check_quantize(activations(3, 512, dtype, 4), ld)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_special_values(dtype):
    t = TYPES[dtype]
    info = torch.finfo(t)
    rows = [torch.zeros(64), torch.full((64,), -0.0), torch.full((64,), info.max), torch.full((64,), info.tiny), torch.full((64,), info.smallest_normal / 2)]
    ties = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 7.5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -7.5])
    rows += [torch.cat((ties * s, torch.zeros(16), ties, ties)) for s in (1.0, 0.5, 4.0)]
    for bad in (float("inf"), -float("inf"), float("nan")):
        r = torch.linspace(-3, 3, 64)
        r[40] = bad
        rows.append(r)
    x = torch.stack(rows).to(t)
    x[4, 1] = torch.tensor(info.smallest_normal * info.eps, dtype=t)         # the smallest subnormal
    x[4, 32:] = torch.tensor(info.smallest_normal * info.eps, dtype=t)
    codes, scales, want_c, want_s = check_quantize(x)
    y = torch.empty((len(rows), 64), dtype=torch.float32, device="cuda")
    sbnn.mxfp4_dequantize(codes, scales, y, 64, len(rows), 64)
    got, want = y.cpu().numpy().astype(np.float64), O.values(want_c, want_s, 64)
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[-3:, 32:]).all() and not np.isnan(got[-3:, :32]).any()
    assert np.array_equal(np.signbit(got[1]), np.ones(64, bool))             # the sign of a zero stays


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,k,ld", [(1, 1, 1), (1, 1000, 1000), (129, 517, 517), (129, 517, 530), (40, 256, 264), (256, 96, 96), (37900, 33, 33), (38000, 64, 64), (37888, 120, 121),
                                    (37889, 128, 128), (9000, 1001, 1001), (4800, 2048, 2056)])
def test_dequantize_is_the_value_rounded_once(m, k, ld, dtype):
    rng = np.random.default_rng(m + k)
    codes = rng.integers(0, 256, (m, 16 * O.blocks_of(k))).astype(np.uint8)
    s = rng.integers(97, 140, (m, O.blocks_of(k))).astype(np.uint8)
    s[0, 0], s[-1, -1] = 0, 255
    want = torch.from_numpy(O.values(codes, s, k)).float().to(TYPES[dtype])        # exact in fp32, so rounded once
    y = torch.full((m, ld), 7.0, dtype=TYPES[dtype], device="cuda")
    sbnn.mxfp4_dequantize(torch.from_numpy(codes).cuda(), torch.from_numpy(O.tile_scales(s, k, 255)).cuda(), y, ld, m, k)
    sbnn.get_async_status()
    got = y.cpu()
    assert torch.equal(got[:, :k].nan_to_num(1e9), want.nan_to_num(1e9)) and bool((got[:, k:] == 7.0).all())


# ---- the layer ----------------------------------------------------------------------------------------

def bound(k, s, y, dtype):
    """Per MMA (64 channels) three terms -- the two blocks' sums, whole multiples of a quarter of their scale, and the accumulator --
    may be cut at 2^-23 of the largest; shares of up to 8 CTAs, the bias and the last rounding come on top."""
    return (3 * -(-k // 64) + 10) * 2.0 ** -23 * s + torch.finfo(TYPES[dtype]).eps / 2 * np.abs(y) * 1.01


def layer(m, k, n, dtype, seed, relu=False, bias=True, ldx=None, ldy=None, pre=False, x=None):
    x = activations(m, k, dtype, seed) if x is None else x
    g = torch.Generator().manual_seed(seed + 1)
    wc, ws = O.quantize((torch.randn((n, k), generator=g) / k ** 0.5).double().numpy())
    b = torch.randn((n,), generator=g) * 0.1 if bias else None
    ldx, ldy = ldx or k, ldy or n
    y = torch.full((m + 2, ldy), 7.0, dtype=TYPES[dtype], device="cuda")
    # rows of no channel get the scale 255: whatever they hold must not matter
    wd, wsd = torch.from_numpy(wc).cuda(), torch.from_numpy(O.tile_scales(ws, k, 255)).cuda()
    bd = b.cuda() if bias else None
    flags = sbnn.SBNN_RELU if relu else 0
    xc, xs = O.quantize(x.double().numpy())
    out = y[1:m + 1]
    if out.data_ptr() % 16:                       # rows of an odd stride: the tensor itself starts on a boundary
        y = torch.full((m + 1, ldy), 7.0, dtype=TYPES[dtype], device="cuda")
        out = y[:m]
    if pre:
        sbnn.conv1x1_mxfp4_q(wd, wsd, bd, torch.from_numpy(xc).cuda(), torch.from_numpy(O.tile_scales(xs, k, 255)).cuda(), out, ldy, m, k, n, flags)
        sbnn.get_async_status()
    else:
        whole, work = guarded(sum(sbnn.mxfp4_bytes(m, k)))
        sbnn.conv1x1_mxfp4(wd, wsd, bd, strided(x, ldx), ldx, out, ldy, m, k, n, flags, work if m > 32 else None)
        sbnn.get_async_status()
        intact(whole)
    ref, s = O.conv1x1(O.values(xc, xs, k), O.values(wc, ws, k), None if b is None else b.numpy(), relu)
    got = out[:, :n].cpu().double().numpy()
    assert bool((out[:, n:] == 7.0).all()) and bool((y[m + 1:] == 7.0).all()), "written outside"
    return got, ref, s


def check_layer(m, k, n, dtype, seed=0, **kw):
    got, ref, s = layer(m, k, n, dtype, seed, **kw)
    worst = np.abs(got - ref) / bound(k, s, ref, dtype)
    assert np.all(worst <= 1), f"worst {worst.max()}"


@pytest.mark.parametrize("m,k,n", [(1, 32, 128), (1, 64, 1), (1, 1, 5), (8, 256, 128), (3, 96, 130), (1, 1024, 1000), (13, 700, 300), (32, 512, 257),
                                   (17, 4096, 64), (2, 8200, 130), (32, 16384, 16), (1, 40000, 40), (32, 65536, 20)])
@pytest.mark.parametrize("pre", [False, True])
def test_few_pixels(m, k, n, pre):
    check_layer(m, k, n, "f32", m + k + n, pre=pre)


@pytest.mark.parametrize("m,k,n", [(32, 10240, 19300), (9, 2000, 40001), (700, 512, 33000)])
def test_many_channels_sampled(m, k, n):
    """Weights that are drawn as codes and scales; some channels of each end and between."""
    g = torch.Generator(device="cuda").manual_seed(k)
    codes = torch.randint(256, (n, 16 * O.blocks_of(k)), generator=g, device="cuda", dtype=torch.uint8)
    if k % 32:
        codes[:, k // 2:] = 0
    scales = torch.randint(118, 124, (sbnn.mxfp4_bytes(n, k)[1],), generator=g, device="cuda", dtype=torch.uint8)
    x = activations(m, k, "bf16", 18)
    y = torch.empty((m, n), device="cuda")
    work = torch.empty((sum(sbnn.mxfp4_bytes(m, k)),), dtype=torch.uint8, device="cuda") if m > 32 else None
    sbnn.conv1x1_mxfp4(codes, scales, None, x.cuda(), k, y, n, m, k, n, 0, work)
    sbnn.get_async_status()
    rows = torch.cat((torch.arange(130), torch.randint(n, (100,), generator=torch.Generator().manual_seed(1)), torch.arange(n - 130, n)))
    off = O.scale_offsets(n, k)[rows]
    wv = O.values(codes[rows.cuda()].cpu().numpy(), scales.cpu().numpy()[off], k)
    xv = O.values(*O.quantize(x.double().numpy()), k)
    ref, s = O.conv1x1(xv, wv, None, False)
    got = y[:, rows.cuda()].cpu().double().numpy()
    assert np.all(np.abs(got - ref) <= bound(k, s, ref, "f32"))


@pytest.mark.parametrize("m,k,n", [(33, 64, 128), (64, 256, 128), (65, 300, 516), (128, 1024, 128), (129, 128, 1000), (196, 517, 516), (500, 2048, 256),
                                   (1000, 96, 2000), (40, 1, 3)])
@pytest.mark.parametrize("pre", [False, True])
def test_more_pixels(m, k, n, pre):
    check_layer(m, k, n, "f32", m + k + n, pre=pre)


@pytest.mark.parametrize("m,k,n", [(1300, 512, 4096), (2500, 384, 4000), (5000, 260, 2050)])
def test_wide_tiles(m, k, n):
    check_layer(m, k, n, "f32", 5)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,k,n", [(1, 1024, 1000), (7, 516, 130), (100, 520, 300)])
@pytest.mark.parametrize("relu", [False, True])
def test_types_and_relu(m, k, n, dtype, relu):
    check_layer(m, k, n, dtype, 11, relu=relu)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [5, 70])
@pytest.mark.parametrize("ldx,ldy", [(300, 205), (301, 200), (312, 208), (305, 203)])
def test_strides(m, ldx, ldy, dtype):
    check_layer(m, 300, 200, dtype, 12, ldx=ldx, ldy=ldy)


@pytest.mark.parametrize("m", [6, 100])
def test_no_bias(m):
    check_layer(m, 256, 128, "f32", 13, bias=False)


@pytest.mark.parametrize("m", [4, 90])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_bad_activations_reach_their_pixel_and_no_other(m, bad):
    k, n = 352, 260
    x = activations(m, k, "f32", 14)
    x[2, 345] = bad
    got, ref, s = layer(m, k, n, "f32", 14, x=x)
    assert np.isnan(got[2]).all()
    keep = np.arange(m) != 2
    assert np.all(np.abs(got - ref)[keep] <= bound(k, s, ref, "f32")[keep])


def test_a_pixel_is_the_same_in_every_place_and_both_entries():
    """Rows are computed alone: the same activations give the same bits in every row of a call, rounded before or inside."""
    for m in (32, 300):
        x = activations(1, 1024, "bf16", 15).expand(m, 1024).contiguous()
        got = [layer(m, 1024, 200, "bf16", 15, x=x, pre=pre)[0] for pre in (False, True)]
        assert np.array_equal(got[0], np.broadcast_to(got[0][:1], got[0].shape)) and np.array_equal(got[0], got[1])


@pytest.mark.parametrize("m,k,n", [(32, 8192, 300), (5, 512, 130), (32, 2000, 19200)])
def test_a_workspace_changes_no_result(m, k, n):
    """Few pixels are rounded by a launch ahead where there is room and that is quicker."""
    g = torch.Generator(device="cuda").manual_seed(k)
    wc, ws = (torch.empty((b,), dtype=torch.uint8, device="cuda") for b in sbnn.mxfp4_bytes(n, k))
    sbnn.mxfp4_quantize(torch.randn((n, k), generator=g, device="cuda"), k, wc, ws, n, k)
    x = torch.randn((m, k), generator=g, device="cuda").half()
    need = sum(sbnn.mxfp4_bytes(m, k))
    got = []
    for size in (None, need - 1, need):
        y = torch.empty((m, n), device="cuda")
        whole, work = guarded(size or 0)
        sbnn.conv1x1_mxfp4(wc, ws, None, x, k, y, n, m, k, n, 0, work if size else None)
        sbnn.get_async_status()
        intact(whole)
        got.append(y)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_results_repeat_bit_by_bit():
    for m, k, n in ((1, 4096, 512), (20, 2048, 1000), (200, 1024, 300)):
        a, b = (layer(m, k, n, "f32", 16)[0] for _ in range(2))
        assert np.array_equal(a, b)


def test_large_and_small_scales():
    """Scales near both ends of their range, products within fp32's."""
    m, k, n = 40, 256, 128
    for ex in (-60, 60):
        x = activations(m, k, "f32", 17) * 2.0 ** ex
        check_layer(m, k, n, "f32", 17, x=x)
        check_layer(3, k, n, "f32", 17, x=x[:3])


@pytest.mark.parametrize("m", [3, 40, 400])
def test_blocks_of_zeros(m):
    """Activations behind a ReLU: blocks, pixels and channels that are zero altogether have the scale 2^-127."""
    x = activations(m, 416, "f32", 19).clamp(min=0)
    x[:, 32:160] = 0
    x[m // 2] = 0
    x[0, 400:] = 2.0 ** -126
    check_layer(m, 416, 260, "f32", 19, x=x, relu=True)


def test_memory_that_is_not_the_devices_is_refused():
    x, y = torch.zeros((2, 64)), torch.zeros((2, 64), device="cuda")
    c, s = torch.zeros((64 * 32,), dtype=torch.uint8, device="cuda"), torch.zeros((512,), dtype=torch.uint8, device="cuda")
    for call in (lambda: sbnn.mxfp4_quantize(x, 64, c, s, 2, 64), lambda: sbnn.mxfp4_dequantize(c.cpu(), s, y, 64, 2, 64),
                 lambda: sbnn.conv1x1_mxfp4(c, s, None, y, 64, x, 64, 2, 64, 64, 0), lambda: sbnn.conv1x1_mxfp4_q(c, s, None, c, s.cpu(), y, 64, 2, 64, 64, 0),
                 lambda: sbnn.logprobs(x, 64, 2, 64, None, 0, None, None, 0, None, None)):
        with pytest.raises(sbnn.SbnnError) as e:
            call()
        assert e.value.name == "SBNN_ERR_CUDA" and "host memory" in e.value.detail
    sbnn.get_async_status()


def test_first_calls_of_a_process_can_be_captured():
    """Nothing is set up by a call outside the capture: a new process records its first calls and replays them."""
    code = """
import torch, paper_2310_19509_b200 as sbnn
x, w = torch.randn((40, 512), device="cuda").bfloat16(), torch.randn((300, 512), device="cuda").bfloat16()
e = lambda n: torch.empty((n,), dtype=torch.uint8, device="cuda")
wc, ws, work = *map(e, sbnn.mxfp4_bytes(300, 512)), e(sum(sbnn.mxfp4_bytes(40, 512)))
y, z = torch.zeros((40, 300), device="cuda"), torch.zeros((3, 300), device="cuda")
h, i, l = torch.zeros((40,), device="cuda"), torch.zeros((40, 3), dtype=torch.int32, device="cuda"), torch.zeros((40, 3), device="cuda")
def calls():
    sbnn.mxfp4_quantize(w, 512, wc, ws, 300, 512)
    sbnn.conv1x1_mxfp4(wc, ws, None, x, 512, y, 300, 40, 512, 300, 0, work)
    sbnn.conv1x1_mxfp4(wc, ws, None, x, 512, z, 300, 3, 512, 300, 0)
    sbnn.logprobs(y, 300, 40, 300, None, 0, None, h, 3, i, l)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    calls()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (y, z, h, i, l)]
calls()
sbnn.get_async_status()
assert all(torch.equal(a, b) for a, b in zip(got, (y, z, h, i, l))) and float(y.abs().sum()) > 0
print("replayed")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert r.returncode == 0 and "replayed" in r.stdout, r.stderr[-2000:]


def test_side_stream_and_graph():
    """A call on another stream, and captured calls with workspaces of their own replayed on new activations."""
    m, k, n = 100, 512, 260
    g = torch.Generator().manual_seed(1)
    w = torch.randn((n, k), generator=g) / 20
    wc, ws = O.quantize(w.double().numpy())
    wd, wsd = torch.from_numpy(wc).cuda(), torch.from_numpy(O.tile_scales(ws, k)).cuda()
    xs = [activations(m, k, "bf16", i).cuda() for i in range(3)]
    x = [torch.empty_like(xs[0]) for _ in range(2)]
    y = [torch.empty((m, n), device="cuda") for _ in range(2)]
    work = [torch.empty((sum(sbnn.mxfp4_bytes(m, k)),), dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = []
    for v in xs:
        sbnn.conv1x1_mxfp4(wd, wsd, None, v, k, y[0], n, m, k, n, 0, work[0])
        want.append(y[0].clone())
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            sbnn.conv1x1_mxfp4(wd, wsd, None, x[i], k, y[i], n, m, k, n, 0, work[i])
    for a, b in ((0, 1), (2, 0), (1, 2)):
        x[0].copy_(xs[a]), x[1].copy_(xs[b])
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(y[0], want[a]) and torch.equal(y[1], want[b])


def test_capture_behind_copies_and_joined_streams():
    """Calls captured behind copies, and behind two streams that join, start when all of that is done."""
    m, k, n = 64, 512, 300
    g = torch.Generator(device="cuda").manual_seed(5)
    w = [torch.randn((n, k), generator=g, device="cuda") for _ in range(3)]
    xs = [torch.randn((m, k), generator=g, device="cuda") for _ in range(3)]
    x, wd, y = torch.zeros_like(xs[0]), torch.zeros_like(w[0]), torch.zeros((m, n), device="cuda")
    wc, ws = (torch.empty((b,), dtype=torch.uint8, device="cuda") for b in sbnn.mxfp4_bytes(n, k))
    work = torch.empty((sum(sbnn.mxfp4_bytes(m, k)),), dtype=torch.uint8, device="cuda")
    h, ti, tl = torch.empty((m,), device="cuda"), torch.empty((m, 4), dtype=torch.int32, device="cuda"), torch.empty((m, 4), device="cuda")
    x_in, w_in = torch.zeros_like(x), torch.zeros_like(wd)
    side = torch.cuda.Stream()

    def calls():
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        x.copy_(x_in)
        with torch.cuda.stream(side):
            wd.copy_(w_in)
            sbnn.mxfp4_quantize(wd, k, wc, ws, n, k)
        here.wait_stream(side)
        sbnn.conv1x1_mxfp4(wc, ws, None, x, k, y, n, m, k, n, 0, work)
        sbnn.logprobs(y, n, m, n, None, 0, None, h, 4, ti, tl)

    want = []
    for a, b in zip(xs, w):
        x_in.copy_(a), w_in.copy_(b)
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        want.append([t.clone() for t in (y, h, ti, tl)])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(5):
        for a, b, expected in zip(xs, w, want):
            x_in.copy_(a), w_in.copy_(b)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip((y, h, ti, tl), expected))


def test_offsets_past_32_bits():
    """The last rows of matrices of more than 2^31 elements."""
    m, k, ld = 70000, 32, 65536
    x = torch.zeros((m * ld,), dtype=torch.bfloat16, device="cuda")
    rows = x.view(m, ld)[:, :k]
    rows.copy_(torch.randn((m, k), generator=torch.Generator().manual_seed(2)).bfloat16().cuda())
    cb, sb = sbnn.mxfp4_bytes(m, k)
    codes, scales = torch.empty((cb,), dtype=torch.uint8, device="cuda"), torch.empty((sb,), dtype=torch.uint8, device="cuda")
    sbnn.mxfp4_quantize(x, ld, codes, scales, m, k)
    want = rows.contiguous().cpu()
    wc, ws = O.quantize(want.double().numpy())
    assert np.array_equal(codes.cpu().numpy().reshape(m, -1), wc)
    sbnn.mxfp4_dequantize(codes, scales, x, ld, m, k)
    assert torch.equal(rows.float().cpu(), torch.from_numpy(O.values(wc, ws, k)).float())
