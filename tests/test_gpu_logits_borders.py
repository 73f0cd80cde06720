"""Borders of top-p that are decided by little: rows in which one weight or its rounding says where the cut is.  And settings at
the ends of their ranges."""

import numpy as np
import pytest
import torch

from oracle import fsd_logits_oracle as lo
from tests import logits as lg

pytestmark = pytest.mark.gpu


def _kept(rows, dtype, top_p, top_k=None):
    """rows: a list a sequence of (value, how many).  How many tokens of each sequence are kept, next to what the oracle keeps."""
    V = max(sum(n for _, n in r) for r in rows)
    c = lg.Call(len(rows), 0, V, dtype, (), seed=40)
    for b, r in enumerate(rows):
        x = torch.cat([torch.full((n,), v, dtype=torch.float64) for v, n in r])
        x = torch.nn.functional.pad(x, (0, V - x.numel()), value=-float("inf"))
        c.logits["target"][b, 0] = x[torch.randperm(V, generator=torch.Generator().manual_seed(b))].to(lg.TORCH[dtype])
    c.o["top_p"] = np.array(top_p, np.float32)
    c.o["top_k"] = None if top_k is None else np.array(top_k, np.int32)
    got = c.run()["target"]
    for b in range(len(rows)):
        y = c.logits["target"][b, 0]
        keep = lo.kept(y.double().numpy(), None if top_k is None else top_k[b], c.o["top_p"][b].item())
        want = torch.where(torch.from_numpy(keep), y, torch.tensor(-float("inf"), dtype=y.dtype))
        assert torch.equal(got[b, 0], want), (b, int((got[b, 0] > -float("inf")).sum()), int(keep.sum()))
    return [int((r > -float("inf")).sum()) for r in got[:, 0]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_share_that_ends_just_behind_many_light_tokens(dtype):
    """The tokens behind a sure one weigh 3e-10 of it each, so that what is missing at the end of some run of values is less than
    1e-9 of the share and is still several tokens."""
    light = [(-13.75, 10), (-13.8125, 1), (-13.875, 316453)]
    assert _kept([[(8.0, 1)] + light], dtype, [0.9999]) == [14]
    rows = [[(8.0, 1), (-13.75, 10), (-13.8125, k), (-13.875, 316453)] for k in range(1, 9)]
    _kept(rows, dtype, [0.9999] * 8)
    _kept(rows, dtype, [0.9999] * 8, [316000] * 8)


TINY = float(torch.tensor([0x33FE], dtype=torch.int16).view(torch.bfloat16).float())       # 1.18e-7


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top_k", [None, 152065])
def test_values_next_to_zero_weigh_what_they_weigh(top_k, dtype):
    """A hundred thousand of 1.18e-7 weigh 0.01 tokens more than as many zeros."""
    rows, share, k = [], [], None
    rows.append([(1.0, 1), (TINY, 100000), (-1.0, 52064)]); share.append(0.8541399836540222)
    rows.append([(1.0, 60000), (-TINY, 92064)]); share.append(0.3000155985355377)
    for p in np.linspace(0.85, 0.97, 14):
        rows.append([(1.0, 1), (TINY, 100000), (-1.0, 52064)]); share.append(p)
    if top_k is not None:
        k = [top_k - 1 - 64 * i for i in range(len(rows))]
    got = _kept(rows, dtype, share, k)
    if top_k is None:
        assert got[:2] == [104821, 28162]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [100, 1000, 8192, 40000])
def test_shares_of_equal_tokens_that_end_on_a_token(n, dtype):
    """Of n equal tokens a share of k / n in 32 bits' fractions keeps k: the predecessors of the next one have the share, not less."""
    values = [0.0625, 0.125, 0.25, -7.8125, -5.875, -3.125, 1.25, 7.5, 12.0, -20.0]
    for p in (0.25, 0.5, 0.75):
        assert _kept([[(v, n)] for v in values], dtype, [p] * len(values)) == [int(p * n)] * len(values)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shares_of_equal_tokens_in_front_of_others(dtype):
    values = [0.0625, 0.125, -7.8125, -5.875, -3.125, 1.25, 7.5, 12.0]
    # some that top_k leaves out, some below all bins, some that weigh e^-40 of the others
    assert _kept([[(v, 1000), (v - 1.0, 5000)] for v in values], dtype, [0.75] * 8, [1000] * 8) == [750] * 8
    assert _kept([[(v, 1000), (v - 1.0, 5000)] for v in values], dtype, [0.75] * 8, [100] * 8) == [75] * 8
    assert _kept([[(v, 1000), (-30000.0, 5000)] for v in values], dtype, [0.75] * 8) == [750] * 8
    assert _kept([[(v, 1000), (v - 40.0, 50)] for v in values], dtype, [0.75] * 8) == [750] * 8


@pytest.mark.parametrize("n", [1000, 30000])
def test_fp32_a_token_behind_equal_ones_that_weighs_next_to_nothing(n):
    """What it adds to the share is n * 5e-14 of a token or more, which double precision tells from nothing and 42 bits do not."""
    values = [1.0, 1.25, 2.5, 3.4375, 0.0625, -3.125]
    rows = [[(v, n), (v - 25.0 + np.log(n / 1000), 4)] for v in values]
    assert _kept(rows, "f32", [0.5] * len(values)) == [n // 2 + 1] * len(values)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps", [("mask", "temp"), ("pen", "bias", "mask", "temp"), ("pen", "mask", "temp", "k", "p", "m"), ("pen", "bias", "mask", "temp", "k", "p", "m")])
def test_masked_tokens_stay_masked_at_any_temperature(steps, dtype):
    """1 / temperature is 0 or infinite at the ends, and its product with -inf or 0 no number."""
    c = lg.Call(4, 2, 1003, dtype, steps, seed=41)
    c.o["temperature"] = np.array([np.inf, 3.4028235e38, 1e-38, 0.5], np.float32)
    got = c.run()
    whole = c.run(c.opts(top_k=None, top_p=None, min_p=None))
    for side, x in whole.items():
        for b in range(4):
            for r in range(x.shape[1]):
                row = lo.context_row(None, side, r)
                off = torch.tensor([not lo.bit(c.o["allowed"][b, row], t) for t in range(c.V)])
                assert (x[b, r][off] == -float("inf")).all() and (got[side][b, r][off] == -float("inf")).all(), (side, b, r)
                assert b != 0 or (x[b, r][~off] == 0).all()
    if "k" in steps:
        c.check_cut(got, whole)
    # A value whose magnitude is 2^128 (1 - 2^-25) or more rounds to infinity in single precision (and in bf16), which the oracle's doubles do not:
    # with a temperature of 1e-38 these are the logits from 3.4 on.  The rest is held to the usual tolerance.  (2^-20 beside the border covers
    # the eight roundings of 2^-24 on the way.)  1 / 3.4e38 is subnormal and off by 2^-150 at most, so |x| times it by |x| 2^-150, less than the 8 * 2^-24 of it that
    # are granted (|x| 1.1 * 2^-149), and the product by TINY.
    far = 2.0 ** 128
    for side, x in whole.items():
        for b in range(4):
            for r in range(x.shape[1]):
                y = x[b, r].double().numpy()
                want, size = c.want(side, b, r)
                over = np.abs(want) > far * (1 + 2.0 ** -20)
                assert np.array_equal(y[over], np.sign(want[over]) * np.inf)
                fin = np.abs(want) < far * (1 - (2.0 ** -20 if dtype == "f32" else 2.0 ** -7))
                may = 8 * 2.0 ** -24 * size[fin] + lg.HALF_STEP[dtype] * (np.abs(want[fin]) + 8 * 2.0 ** -24 * size[fin]) + lg.TINY[dtype]
                assert (np.abs(y[fin] - want[fin]) <= may).all(), (side, b, r)
