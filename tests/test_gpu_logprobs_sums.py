"""Sums of long rows of logits, to what their own additions cost and no more: no vector is lost at the end of a share."""
import numpy as np
import pytest
import torch

import paper_2310_19509_b200 as sbnn
from oracle import mxfp4 as O
from test_gpu_logprobs import TYPES, logits, run

pytestmark = pytest.mark.gpu
E = 2.0 ** -24                       # half a step of fp32


def additions(rows, v, ld, dtype, top):
    """(terms that one accumulator takes one after the other, times that a larger base can come) at most, by how rows are dealt out:
    a thread adds its vectors up in pairs, and what it does not hold arrives in groups of four vectors."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    per = 4 if dtype == "f32" else 8
    vectors = (v + (1 if ld % per == 0 else 2) * (per - 1)) // per
    if vectors <= 256:
        return 8 * per // 2, 1       # held by a warp or more
    parts = 1
    while parts < 8 and rows * parts * 2 <= 2 * sms and vectors // (parts * 2) >= 256:
        parts *= 2
    share = -(-vectors // parts)
    held = -(-share // 256)
    return max(8, held) * per // 2, max(1, held // 4 + 6)


def bounds(x, lp, h, ld, dtype, top):
    """What log probabilities and entropy may be off by, per row: [rows][1] beside |lp|, and [rows].

    t is off by 2 E |t| (its own rounding and that of log2 e; the rounding of the base is in every term and in the answer's t alike).
    s: `terms` additions and 4 + 9 + 3 + 7 joins of E each; an exponential is off by 4 E (ex2.approx) and by what its argument is; every new base brings an exponential, its argument and two products, 7 E.  Joins bring three more bases at most.
    log2 is off by an ulp, 2 E; differences, products and ln 2 itself by E each."""
    rows, v = x.shape
    terms, bases = additions(rows, v, ld, dtype, top)
    t = (x - x.max(axis=1, keepdims=True)) / np.log(2)
    p = np.exp2(t)
    p /= p.sum(axis=1, keepdims=True)
    far, far2 = (p * np.abs(t)).sum(axis=1), (p * t * t).sum(axis=1)
    log2_s = -t.max(axis=1) + np.log2(np.exp2(t).sum(axis=1))
    rel = (terms + 23 + 4 + 7 * (bases + 3)) * E + 2 * np.log(2) * far * E
    on_lp = rel + np.log(2) * log2_s * 4 * E
    on_h = rel + np.log(2) * (far * (2 * rel + 4 * E) + 2 * far2 * E + log2_s * 2 * E + 4 * (bases + 3) * E) + 4 * E * np.abs(h)
    return on_lp[:, None], on_h


def check(x, dtype, targets, top, ld=None):
    """x: fp32 values that the type holds."""
    ld = ld or x.shape[1]
    x = x.to(TYPES[dtype])
    got, want = run(x, targets, top, ld), O.logprobs(x.double().numpy(), targets.numpy(), top)
    on_lp, on_h = bounds(x.double().numpy(), want[0], want[1], ld, dtype, top)
    assert np.array_equal(got[2], want[2])
    for g, w in ((got[0], want[0]), (got[3], want[3])):
        worst = np.abs(g - w) / (on_lp + 5 * E * np.abs(w))
        assert np.all(worst <= 1), f"log probabilities: {worst.max()} of the bound"
    worst = np.abs(got[1] - want[1]) / on_h
    assert np.all(worst <= 1), f"entropy: {worst.max()} of the bound"


# By a warp, by 128, 256 and 512 threads that hold a row, by a cluster that holds it or streams it, by a CTA that streams it.
ROWS = [(1250, 600), (400, 2600), (120, 5000), (200, 16001), (3, 5000), (5, 24001), (300, 20000), (160, 50257), (2, 131072), (40, 131073), (1, 262144)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v", ROWS)
@pytest.mark.parametrize("odd", [0, 1])
def test_equal_logits(rows, v, dtype, odd):
    t = torch.tensor([[0, v // 2, v - 1]]).expand(rows, -1).contiguous()
    check(torch.full((rows, v), -1.5), dtype, t, 1, v + odd)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v", ROWS)
@pytest.mark.parametrize("odd", [0, 1])
def test_zeros_are_counted(rows, v, dtype, odd):
    """The exponential of 0 is 1 exactly and a count of such is, too: what is left is the logarithm (an ulp, 2 E), ln 2 and a product
    (E each).  A lost vector, or half of one, is far more."""
    t = torch.tensor([[0, v // 2, v - 1]]).expand(rows, -1).contiguous()
    lp, h, ti, tl = run(torch.zeros((rows, v)).to(TYPES[dtype]), t, 2, v + odd)
    off = 4 * E * np.log(v)
    assert off < 1 / v
    for got in (lp, tl, -h):
        assert np.all(np.abs(got + np.log(v)) <= off)
    assert np.array_equal(ti, np.tile([0, 1], (rows, 1)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v", ROWS)
@pytest.mark.parametrize("odd", [0, 3])
def test_weight_at_the_ends_of_shares(rows, v, dtype, odd):
    """Nearly all of the probability lies in classes where a row can be divided: its ends, the ends of its parts, of the first
    vectors of the threads and of the groups that they stream."""
    per = 4 if dtype == "f32" else 8
    at = {0, 1, v - 1, v - 2}
    for parts in (2, 4, 8):
        for q in range(1, parts):
            at |= {v * q // parts + d for d in range(-2 * per, 2 * per + 1)}
    for step in (32 * per, 128 * per, 256 * per, 512 * per, 1024 * per):
        for q in (1, 2, 3, (v - 1) // step):
            at |= {q * step + d for d in (-per - 1, -per, -1, 0, 1, per - 1, per)}
    at |= {v - d for d in range(1, 8 * per)}
    at = torch.tensor(sorted(a for a in at if 0 <= a < v))
    x = logits(rows, v, dtype, 31, 1.0).float()
    x[:, at] = 14.0 + torch.randint(3, (rows, len(at)), generator=torch.Generator().manual_seed(v)) / 4
    targets = at[torch.randint(len(at), (rows, 4), generator=torch.Generator().manual_seed(rows))]
    check(x, dtype, targets, 8, v + odd)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,v", ROWS)
@pytest.mark.parametrize("order", ["drawn", "rising"])
def test_drawn_and_rising_rows(rows, v, dtype, order):
    """Rising rows bring a larger base with every vector."""
    x = logits(rows, v, dtype, rows, 3.0).float()
    if order == "rising":
        x = x.sort(dim=1).values
    targets = torch.randint(v, (rows, 3), generator=torch.Generator().manual_seed(v))
    check(x, dtype, targets, 20)


@pytest.mark.parametrize("rows,v", ROWS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("around", [1e6, -1e6])
def test_logits_around_a_million(rows, v, dtype, around):
    """Beyond a million differences are taken before they are scaled: shares of a row lie on either side, some far below."""
    step = 0.0625 if dtype == "f32" else 4096.0
    g = torch.Generator().manual_seed(v)
    x = around + step * torch.randint(-40, 41, (rows, v), generator=g).float()
    x[:, : v // 3] -= 50 * step                       # the first third below the border, or further below it
    x[:, v // 2::97] = around * 3 if around < 0 else -around
    targets = torch.randint(v, (rows, 3), generator=g)
    check(x, dtype, targets, 8)
