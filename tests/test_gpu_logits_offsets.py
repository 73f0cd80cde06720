"""Offsets of ragged lists up to the largest 32-bit number.  The lists themselves are short: only entries between a sequence's two
offsets are read, so that a list may stand for the last few thousand entries of a very long one."""

import numpy as np
import pytest
import torch

import paper_2502_20704_b200 as fsd
from oracle import fsd_logits_oracle as lo
from tests import logits as lg

pytestmark = pytest.mark.gpu
END = 2 ** 31 - 1


def _late(flat):
    """A tensor and the address that entry 0 would have if the tensor's last entry were entry END - 1."""
    t = lg.dev(flat)
    return t, t.data_ptr() - 4 * (END - t.numel())


def test_counts_of_lists_that_end_at_the_largest_offset():
    V, rng = 700, np.random.default_rng(1)
    lengths = [5000, 0, 3, 1500]
    prompts = [rng.integers(0, V, n).tolist() for n in lengths]
    outputs = [rng.integers(0, V, n).tolist() for n in reversed(lengths)]
    state = []
    keep = []
    for lists in (prompts, outputs):
        flat = np.concatenate([np.array(x, np.int32) for x in lists])
        t, address = _late(flat)
        offsets = lg.dev((END - flat.size + np.concatenate([[0], np.cumsum([len(x) for x in lists])])).astype(np.int32))
        keep.append((t, offsets))
        state += [offsets, address]
    counts = torch.full((4, V), -7, dtype=torch.int32, device="cuda")
    seen = torch.full((4, (V + 31) // 32), -7, dtype=torch.int32, device="cuda")
    assert fsd.fsd_history_build(*state, 4, V, counts, seen, torch.cuda.current_stream().cuda_stream) == 0
    want = lo.build(prompts, outputs, V)
    assert np.array_equal(counts.cpu().numpy(), want[0]) and np.array_equal(seen.cpu().numpy().view(np.uint32), want[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_biases_that_end_at_the_largest_offset(dtype):
    c = lg.Call(4, 1, 3000, dtype, ("bias",), seed=60)
    rng = np.random.default_rng(2)
    lengths = np.array([400, 0, 2, 300])
    n = int(lengths.sum())
    c.o["bias_tokens"], c.o["bias_values"] = rng.integers(0, 3000, n).astype(np.int32), rng.standard_normal(n).astype(np.float32)
    c.o["bias_offsets"] = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    (t, at), (v, av) = _late(c.o["bias_tokens"]), _late(c.o["bias_values"])
    late = fsd.make_process_opts(dtype=dtype, bias_offsets=lg.dev((c.o["bias_offsets"].astype(np.int64) + END - n).astype(np.int32)), bias_tokens=at, bias_values=av)
    c.check_values(c.run(late))
