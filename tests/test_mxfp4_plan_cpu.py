"""What 4-bit layers run on, decided on the host: plans fit the device, and calls that none fits are refused.  No GPU."""
import numpy as np
import pytest

import paper_2310_19509_b200 as sbnn
from test_mxfp4_cpu import P, T, name

ROOM = 227 * 1024      # shared memory that a CTA may have


@pytest.mark.parametrize("k", [108 * 10 ** 6, 2 ** 28, 805306368, 2 ** 30 - 5, 2 ** 30])
@pytest.mark.parametrize("m", [1, 9, 24, 32])
@pytest.mark.parametrize("n", [1, 128, 20000])
def test_activations_that_no_shared_memory_holds_are_rounded_ahead(m, k, n):
    """A CTA's share of such rows is more than 2^31 bytes in 4 bits, or a multiple of 2^32 and a little."""
    for given in (0, 2):
        pair, pixels, split, rounds, shared = sbnn.debug_plan_conv1x1_mxfp4(m, k, n, activations=given)
        assert not pair and not rounds and pixels == (m + 7) // 8 * 8 and 1 <= split <= 8 and 0 < shared <= ROOM
    with pytest.raises(sbnn.SbnnError) as e:
        sbnn.debug_plan_conv1x1_mxfp4(m, k, n, activations=1)
    assert e.value.name == "SBNN_ERR_NULL"


def test_wide_rows_without_a_workspace_are_refused_before_any_device_is_asked():
    for m, k in ((1, 2 ** 20), (1, 2 ** 28), (24, 805306368), (32, 2 ** 30)):
        need = sum(sbnn.mxfp4_bytes(m, k))
        for work in (None, T("uint8", nbytes=need - 1), T("uint8", at=P + 8, nbytes=need)):
            assert name(sbnn.conv1x1_mxfp4, P, P, None, T(), k, T(), 48, m, k, 48, 0, work) == "SBNN_ERR_NULL"


def test_rows_up_to_the_documented_width_need_no_workspace():
    for m in (1, 8, 17, 32):
        for k in (1, 256, 4096, 40000, 65536):
            for n in (1, 1000, 128 * 148, 128 * 149, 128 * 296, 128 * 297, 2 ** 20):
                pair, pixels, split, rounds, shared = sbnn.debug_plan_conv1x1_mxfp4(m, k, n, activations=1)
                assert rounds and not pair and 0 < shared <= ROOM


def test_few_pixels_are_summed_alike_by_every_entry():
    """The CTAs that share a tile decide the order of its sums: the same however the activations come."""
    rng = np.random.default_rng(0)
    for _ in range(300):
        m, k, n = int(rng.integers(1, 33)), int(2 ** rng.uniform(0, 22)), int(2 ** rng.uniform(0, 18))
        plans = [sbnn.debug_plan_conv1x1_mxfp4(m, k, n, activations=given) for given in (0, 2)]
        try:
            plans.append(sbnn.debug_plan_conv1x1_mxfp4(m, k, n, activations=1))
        except sbnn.SbnnError:
            assert k > 65536
        assert len({p[:3] for p in plans}) == 1 and all(0 < p[4] <= ROOM for p in plans)


def test_plans_of_any_size_fit():
    rng = np.random.default_rng(1)
    for _ in range(2000):
        m, k, n = (int(2 ** rng.uniform(0, 30)) for _ in range(3))
        for y_type in (sbnn.SBNN_F32, sbnn.SBNN_BF16):
            pair, pixels, split, rounds, shared = sbnn.debug_plan_conv1x1_mxfp4(m, k, n, y_type, 2, int(rng.integers(2, 160)))
            assert pixels and 1 <= split <= 8 and (shared == 0 if pair else 0 < shared <= ROOM)


def test_plan_refusals():
    def plan(*a):
        with pytest.raises(sbnn.SbnnError) as e:
            sbnn.debug_plan_conv1x1_mxfp4(*a)
        return e.value.name

    assert plan(0, 8, 8) == plan(4, 0, 8) == plan(4, 8, 8, 0, 3) == plan(4, 8, 8, 0, 2, 0) == plan(40, 8, 8, 0, 2, 1) == plan(40, 8, 8, 0, 2, 2 ** 31 - 1) == "SBNN_ERR_SHAPE"
    assert plan(4, 2 ** 30 + 1, 8) == plan(4, 8, 8, 9) == "SBNN_ERR_UNSUPPORTED"


def test_sizes_of_rows_that_no_call_takes_are_refused():
    """(Sums of channels and a block's or a tile's rounding pass 2^31 for the last of these.)"""
    assert sbnn.mxfp4_bytes(1, 2 ** 30) == (2 ** 29, 512 * 2 ** 23)
    for k in (2 ** 30 + 1, 2 ** 31 - 128, 2 ** 31 - 32, 2 ** 31 - 1):
        for m in (0, 1, 1000):
            with pytest.raises(sbnn.SbnnError) as e:
                sbnn.mxfp4_bytes(m, k)
            assert e.value.name == "SBNN_ERR_UNSUPPORTED"


def test_the_smoke_test_runs_every_kernel_of_the_layer():
    from __graft_entry__ import FOUR_BIT_LAYERS

    plans = [sbnn.debug_plan_conv1x1_mxfp4(*layer) for layer in FOUR_BIT_LAYERS]
    assert [p[3] for p in plans] == [True, False, False] and [p[0] for p in plans] == [False, False, True]
