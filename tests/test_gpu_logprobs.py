"""Log probabilities, entropy and most probable classes against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2310_19509_b200 as sbnn
from oracle import mxfp4 as O

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def run(x, targets, top, ld=None, entropy=True):
    """x [rows][v] on the CPU; returns numpy arrays (log probabilities, entropy, indexes, their log probabilities)."""
    rows, v = x.shape
    ld = ld or v
    buf = torch.full((rows, ld), 1e4, dtype=x.dtype, device="cuda")           # what is between the rows must not count
    buf[:, :v] = x.cuda()
    nt = targets.shape[1]
    lp, h = torch.full((rows + 1, max(nt, 1)), 7.0, device="cuda"), torch.full((rows + 1,), 7.0, device="cuda")
    ti, tl = torch.full((rows + 1, max(top, 1)), -7, dtype=torch.int32, device="cuda"), torch.full((rows + 1, max(top, 1)), 7.0, device="cuda")
    sbnn.logprobs(buf, ld, rows, v, targets.int().cuda() if nt else None, nt, lp if nt else None, h if entropy else None, top,
                  ti if top else None, tl if top else None)
    sbnn.get_async_status()
    assert bool((lp.view(-1)[rows * nt:] == 7).all()) and bool((ti.view(-1)[rows * top:] == -7).all()) and float(h[rows]) == 7.0
    return (lp.view(-1)[:rows * nt].view(rows, nt).cpu().double().numpy(), h[:rows].cpu().double().numpy(),
            ti.view(-1)[:rows * top].view(rows, top).cpu().numpy(), tl.view(-1)[:rows * top].view(rows, top).cpu().double().numpy())


def check(x, targets=None, top=5, ld=None):
    rows, v = x.shape
    if targets is None:
        targets = torch.randint(v, (rows, 2), generator=torch.Generator().manual_seed(rows + v))
    top = min(top, v)
    got, want = run(x, targets, top, ld), O.logprobs(x.double().numpy(), targets.numpy(), top)
    assert np.array_equal(got[2], want[2])
    # A thread adds up to v / 32 exponentials one by one; each is off by at most 2^-21 (two rounded steps and the approximation),
    # far ones by |d| 2^-23 of next to nothing; joins and the logarithm add a few more roundings.
    rel = (v / 32 + 64) * 2.0 ** -24 + 2.0 ** -20
    for g, w in ((got[0], want[0]), (got[3], want[3])):
        assert np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(np.isinf(g), np.isinf(w))
        f = np.isfinite(w)
        assert np.all(np.abs(g[f] - w[f]) <= rel + 4 * 2.0 ** -24 * np.abs(w[f]))
    f = np.isfinite(want[1])
    assert np.array_equal(np.isnan(got[1]), np.isnan(want[1]))
    assert np.all(np.abs(got[1][f] - want[1][f]) <= rel * (2 + 4 * np.abs(want[1][f])))


def logits(rows, v, dtype, seed=0, scale=2.5):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn((rows, v), generator=g)).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v", [(1, 1), (3, 2), (2, 7), (5, 33), (4, 100), (64, 1000), (3, 1024), (2, 4099), (7, 8192), (5, 16500), (1, 50257),
                                    (2, 131072), (200, 9001), (1300, 10), (1250, 1000), (1200, 2000), (400, 1253),
                                    (350, 4100), (300, 8100)])
def test_sizes(rows, v, dtype):
    check(logits(rows, v, dtype, rows + v))


@pytest.mark.parametrize("top", [0, 1, 2, 20, 31, 32])
@pytest.mark.parametrize("rows,v", [(1300, 300), (700, 422), (4, 302), (3, 32), (3, 3000), (2, 40000), (300, 20000), (400, 2600)])
def test_numbers_of_alternatives(rows, v, top):
    check(logits(rows, v, "bf16", top), top=top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("v,ld", [(1000, 1001), (1000, 1003), (517, 530), (20001, 20003), (5, 9)])
@pytest.mark.parametrize("rows", [9, 1250])
def test_strides(rows, v, ld, dtype):
    if rows * ld > 5e6:
        rows = 200
    check(logits(rows, v, dtype, 3), ld=ld)


# One size for every form a row is worked on in: by a warp, a cluster of CTAs that hold it, CTAs that stream it, that hold it.
SHAPES = [(1250, 600), (3, 1000), (300, 20000), (2, 70001), (320, 3001)]


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_logits_go_by_index(rows, v, dtype):
    check(torch.full((rows, v), -1.5).to(TYPES[dtype]), top=32)
    x = torch.zeros((rows, v))
    x[:, v // 3::7] = 2.0                                        # thousands of classes share the largest value
    check(x.to(TYPES[dtype]), top=32)
    x = torch.zeros((rows, v))
    x[:, 0::2] = -0.0                                            # zeros of both signs are equal
    check(x.to(TYPES[dtype]), top=20)


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_masked_rows(rows, v, dtype):
    x = logits(rows, v, dtype, 4)
    allowed = [0, 1, 5, v // 2, v]
    for r in range(rows):
        keep = allowed[r % 5]
        if keep < v:
            gone = torch.randperm(v, generator=torch.Generator().manual_seed(r))[keep:]
            x[r, gone] = -float("inf")
    check(x, top=8)
    low = torch.where(torch.isinf(x), torch.full_like(x, torch.finfo(x.dtype).min), x)
    check(low, top=8)                                            # masks of the type's lowest value; rows of nothing else are uniform


@pytest.mark.parametrize("rows,v", SHAPES)
def test_one_class_that_is_not_masked_is_certain(rows, v):
    x = torch.full((rows, v), -float("inf"))
    x[torch.arange(rows), torch.arange(rows) * 37 % v] = torch.finfo(torch.float32).min
    got = run(x, (torch.arange(rows) * 37 % v)[:, None], 2)
    assert np.all(got[0] == 0) and np.all(got[1] == 0) and np.array_equal(got[2][:, 0], (np.arange(rows) * 37) % v)
    assert np.all(np.isneginf(got[3][:, 1]))


@pytest.mark.parametrize("rows,v", SHAPES)
def test_infinities_and_nan(rows, v):
    x = logits(rows, v, "f32", 5)
    x[0, v // 2] = float("nan")
    x[1, 3], x[1, v - 1] = float("inf"), float("inf")
    if rows > 2:
        x[2] = float("nan")
    check(x, top=6)


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("order", ["falling", "rising", "blocks"])
def test_logits_in_order(rows, v, order):
    """Rows whose largest classes crowd in one place, or come round with the period that threads go by."""
    x = torch.arange(v, 0, -1, dtype=torch.float32) / 64
    if order == "rising":
        x = x.flip(0)
    if order == "blocks":
        x = ((torch.arange(v) // 8 % 128 == 5).float() * 4 + torch.arange(v) % 4096 / 4096)
    check(x.expand(rows, v).contiguous(), top=32)


@pytest.mark.parametrize("rows,v", SHAPES)
def test_targets(rows, v):
    t = torch.tensor([0, v - 1, -1, -100, v, v + 5, 2 ** 31 - 1, -2 ** 31, 1])
    check(logits(rows, v, "f16", 6), targets=t.expand(rows, -1).contiguous())
    check(logits(rows, v, "f16", 6), targets=torch.zeros((rows, 0)), top=3)


def test_large_magnitudes():
    x = logits(20, 3000, "f32", 7) * 1e37                         # differences beyond the range of exponentials
    check(x, top=4)
    check(logits(20, 3000, "f32", 7) + 1e4, top=4)


def test_results_repeat_and_graph():
    x = logits(2, 131072, "bf16", 8).cuda()
    t = torch.tensor([[5], [77]], dtype=torch.int32, device="cuda")
    outs = [(torch.empty((2, 1), device="cuda"), torch.empty((2,), device="cuda"), torch.empty((2, 20), dtype=torch.int32, device="cuda"),
             torch.empty((2, 20), device="cuda")) for _ in range(2)]

    def call(o):
        sbnn.logprobs(x, 131072, 2, 131072, t, 1, o[0], o[1], 20, o[2], o[3])

    call(outs[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(outs[1])
    for _ in range(3):
        for o in outs[1]:
            o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_row_offsets_past_32_bits():
    rows, v, ld = 40000, 10, 65536
    x = torch.zeros((rows * ld,), dtype=torch.bfloat16, device="cuda")
    x.view(rows, ld)[:, :v] = logits(rows, v, "bf16", 9).cuda()
    h, ti, tl = torch.empty((rows,), device="cuda"), torch.empty((rows, 2), dtype=torch.int32, device="cuda"), torch.empty((rows, 2), device="cuda")
    sbnn.logprobs(x, ld, rows, v, None, 0, None, h, 2, ti, tl)
    want = O.logprobs(x.view(rows, ld)[:, :v].double().cpu().numpy(), np.zeros((rows, 0)), 2)
    assert np.array_equal(ti.cpu().numpy(), want[2])
    assert np.all(np.abs(h.cpu().double().numpy() - want[1]) <= 1e-5)


def test_classifier_head_in_4_bits_and_its_answers():
    """Features -> 4-bit classifier -> answers, as they are used: the answers are those of the logits that the layer gave."""
    m, k, n = 64, 1024, 1000
    g = torch.Generator().manual_seed(3)
    x, w, b = torch.randn((m, k), generator=g).cuda(), (torch.randn((n, k), generator=g) / 8).cuda(), torch.randn((n,), generator=g).cuda()
    cb, sb = sbnn.mxfp4_bytes(n, k)
    wc, ws = torch.empty((cb,), dtype=torch.uint8, device="cuda"), torch.empty((sb,), dtype=torch.uint8, device="cuda")
    sbnn.mxfp4_quantize(w, k, wc, ws, n, k)
    work = torch.empty((sum(sbnn.mxfp4_bytes(m, k)),), dtype=torch.uint8, device="cuda")
    y = torch.empty((m, n), device="cuda")
    lp, h, ti, tl = (torch.empty((m,), device="cuda"), torch.empty((m,), device="cuda"), torch.empty((m, 5), dtype=torch.int32, device="cuda"),
                     torch.empty((m, 5), device="cuda"))
    t = torch.randint(n, (m,), generator=g).int().cuda()
    sbnn.conv1x1_mxfp4(wc, ws, b, x, k, y, n, m, k, n, 0, work)
    sbnn.logprobs(y, n, m, n, t, 1, lp, h, 5, ti, tl)
    sbnn.get_async_status()
    want = O.logprobs(y.double().cpu().numpy(), t.cpu().numpy(), 5)
    assert np.array_equal(ti.cpu().numpy(), want[2])
    for got, ref in ((lp.view(-1, 1), want[0]), (h, want[1]), (tl, want[3])):
        assert np.all(np.abs(got.cpu().double().numpy() - ref) <= 1e-5 + 1e-6 * np.abs(ref))
    vx, vw = (O.values(*O.quantize(v.double().cpu().numpy()), k) for v in (x, w))
    ref, s = O.conv1x1(vx, vw, b.cpu().numpy(), False)
    assert np.all(np.abs(y.cpu().double().numpy() - ref) <= (3 * 16 + 10) * 2.0 ** -23 * s + 2.0 ** -24 * np.abs(ref))
