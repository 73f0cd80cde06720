"""Logit processing, truncation and token counts on the GPU against their oracle, through the C ABI."""

import numpy as np
import pytest
import torch

import paper_2502_20704_b200 as fsd
from oracle import fsd_logits_oracle as lo
from oracle import fsd_oracle as orc
from tests import logits as lg

pytestmark = pytest.mark.gpu
CUT = {"top_k": None, "top_p": None, "min_p": None}


# ---- penalties, biases, masks, temperature -----------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,V", [(1, 0, 1), (2, 1, 2), (1, 3, 7), (3, 2, 31), (2, 4, 33), (1, 0, 1000), (3, 2, 2049), (2, 5, 4099), (2, 3, 8192), (1, 2, 20011)])
def test_chain_rows(B, P, V, dtype):
    c = lg.Call(B, P, V, dtype)
    c.check_values(c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps", [(), ("pen",), ("bias",), ("mask",), ("temp",), ("pen", "temp"), ("bias", "mask")])
def test_each_step_alone(steps, dtype):
    c = lg.Call(3, 3, 1501, dtype, steps, seed=1)
    c.check_values(c.run())


@pytest.mark.parametrize("only", ["repetition", "frequency", "presence"])
def test_each_penalty_alone(only):
    c = lg.Call(3, 3, 500, "f32", ("pen",), seed=2)
    for k in ("repetition", "frequency", "presence"):
        if k != only:
            c.o[k] = None
    c.check_values(c.run())


def test_drafted_tokens_count_without_a_history_and_a_history_without_drafted_tokens():
    c = lg.Call(3, 4, 300, "f32", ("pen",), seed=3)
    c.check_values(c.run(tokens=None), tokens=False)
    c.o["counts"] = c.o["seen"] = None
    c.check_values(c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lead_in,lead_out", [(1, 1), (3, 0), (0, 5), (7, 2)])
@pytest.mark.parametrize("V", [513, 2048])
def test_rows_off_the_boundaries(V, lead_in, lead_out, dtype):
    c = lg.Call(2, 2, V, dtype, seed=4)
    c.check_values(c.run(lead=(lead_in, lead_out)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps", [("pen", "bias", "mask", "temp"), ("pen", "temp", "k", "p", "m")])
@pytest.mark.parametrize("lead", [0, 3])
def test_in_place_is_the_same(lead, steps, dtype):
    c = lg.Call(2, 3, 3001, dtype, steps, seed=5)
    a, b = c.run(lead=(lead, lead)), c.run(in_place=True, lead=(lead, lead))
    assert all(torch.equal(a[s].view(torch.uint8), b[s].view(torch.uint8)) for s in a)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,V", [(1, 1, 40), (2, 9, 777), (1, 40, 4096)])
def test_tree_rows(B, N, V, dtype):
    c = lg.Call(B, N, V, dtype, call="tree", seed=6)
    c.check_values(c.run())


def test_a_tree_with_parents_out_of_range():
    c = lg.Call(2, 8, 100, "f32", call="tree", seed=7)
    c.parent[0] = [5, -7, 1, 3, 2, 99, 5, 7]
    c.check_values(c.run())


def test_a_chain_is_a_tree_of_one_branch():
    c = lg.Call(2, 6, 900, "f32", seed=8)
    a = c.run()
    c.call, c.parent = "tree", np.tile(np.arange(-1, 5, dtype=np.int32), (2, 1))
    b = c.run()
    assert all(torch.equal(a[s], b[s]) for s in a)


def test_drafted_and_biased_ids_outside_the_vocabulary_and_ids_named_twice():
    c = lg.Call(2, 4, 65, "f32", seed=9)
    c.tokens[0] = [-1, 65, 3, 3]
    c.tokens[1] = [2 ** 31 - 1, -2 ** 31, 64, 64]
    c.o["bias_offsets"] = np.array([0, 5, 9], np.int32)
    c.o["bias_tokens"] = np.array([3, 64, 3, 65, -1, 0, 0, 0, 2 ** 31 - 1], np.int32)
    c.o["bias_values"] = np.arange(1, 10, dtype=np.float32)
    c.check_values(c.run())


def test_bias_lists_that_are_empty_or_hold_the_whole_vocabulary():
    c = lg.Call(3, 1, 5000, "f32", seed=10)
    rng = np.random.default_rng(3)
    c.o["bias_offsets"] = np.array([0, 0, 5000, 5000], np.int32)
    c.o["bias_tokens"] = rng.permutation(5000).astype(np.int32)
    c.o["bias_values"] = rng.standard_normal(5000).astype(np.float32)
    c.check_values(c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_stands_in_masked_places_does_not_matter(dtype):
    c = lg.Call(2, 2, 1000, dtype, ("mask", "temp"), seed=11)
    a = c.run()
    for side, x in c.logits.items():
        for r in range(x.shape[1]):
            for b in range(2):
                off = torch.tensor([not lo.bit(c.o["allowed"][b, r], t) for t in range(1000)])
                junk = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(x.dtype).min]).to(x.dtype).repeat(250)
                x[b, r] = torch.where(off, junk, x[b, r])
    b = c.run()
    assert all(torch.equal(a[s].view(torch.uint8), b[s].view(torch.uint8)) for s in a)


def test_masks_that_leave_nothing_and_values_that_are_not_finite():
    c = lg.Call(3, 1, 257, "f32", ("pen", "mask", "temp"), seed=12)
    c.o["allowed"][0] = 0
    c.o["allowed"][1] = 0xFFFFFFFF
    x = c.logits["target"]
    x[1, 0, 5], x[1, 0, 6], x[1, 0, 7], x[1, 1, 8] = float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min
    got = c.run()
    assert (got["target"][0] == -float("inf")).all()
    c.check_values(got)


def test_temperatures_that_are_no_temperature_leave_the_row_undivided():
    c = lg.Call(4, 0, 100, "f32", ("temp",), seed=13)
    c.o["temperature"] = np.array([0.0, -1.0, np.nan, 2.0], np.float32)
    got = c.run()["target"]
    assert torch.equal(got[:3], c.logits["target"][:3]) and torch.equal(got[3], c.logits["target"][3] / 2)


# ---- top-k, top-p, min-p -------------------------------------------------------------------------
def _cut(c, **kw):
    got = c.run(**kw)
    c.check_cut(got, c.run(c.opts(**CUT)))
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("steps", [("k",), ("p",), ("m",), ("k", "p"), ("k", "p", "m"), ("pen", "bias", "mask", "temp", "k", "p", "m")])
@pytest.mark.parametrize("B,P,V", [(4, 1, 1), (6, 1, 2), (6, 1, 9), (8, 2, 100), (12, 1, 1031), (8, 1, 5000)])
def test_cut_rows(B, P, V, steps, dtype):
    _cut(lg.Call(B, P, V, dtype, steps, seed=20))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [32000, 50257, 128256, 256000, 800001])
def test_cut_long_rows(V, dtype):
    c = lg.Call(6, 0, V, dtype, ("temp", "k", "p", "m"), seed=21)
    c.o["top_k"] = np.array([0, 0, 50, V // 3, 0, 1000], np.int32)
    c.o["top_p"] = np.array([0.9, 1.0, 0.95, 0.7, 0.999, 0.5], np.float32)
    c.o["min_p"] = np.array([0.0, 0.02, 0.0, 0.0, 1e-6, 0.0], np.float32)
    _cut(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["flat", "one", "two_values", "zeros", "far", "huge", "tiny", "ramp", "mostly_masked", "narrow"])
def test_cut_rows_of_every_shape(shape, dtype):
    V, B = 40000, 8
    c = lg.Call(B, 0, V, dtype, ("k", "p", "m"), seed=22)
    c.o["top_k"] = np.array([0, 0, 0, 7, 5000, 39999, 20000, 0], np.int32)
    c.o["top_p"] = np.array([0.5, 0.9, 0.001, 1.0, 0.9, 0.75, 0.3, 1.0], np.float32)
    c.o["min_p"] = np.array([0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 1e-3, 0.01], np.float32)
    x, g = c.logits["target"], torch.Generator().manual_seed(4)
    t = torch.arange(V, dtype=torch.float32)
    n = torch.randn(B, 1, V, generator=g)
    x.copy_({"flat": torch.full((B, 1, V), -3.25), "one": torch.where(t == 777, 50.0, -50.0).expand(B, 1, V), "two_values": torch.where(n > 1, 1.0, 0.5),
             "zeros": torch.where(n > 0, 0.0, -0.0), "far": n * 200 - 3000, "huge": n * 1e30, "tiny": n * 1e-6, "ramp": -t.expand(B, 1, V) * 1e-3,
             "mostly_masked": torch.where(n > 3.0, n, torch.tensor(-float("inf"))), "narrow": 7 + n * 0.01}[shape])
    _cut(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,share", [(100003, 0.02), (100003, 0.6), (60000, 1.0), (300001, 0.01)])
def test_cut_long_rows_of_long_histories(V, share, dtype):
    """Few and many used ids, drafted ones, penalties that lower and that raise."""
    c = lg.Call(4, 2, V, dtype, ("pen", "temp", "k", "p", "m"), seed=29)
    rng = np.random.default_rng(V)
    used = rng.random((4, V)) < share
    c.o["seen"], c.o["counts"] = lg.bits_of(used), (used * rng.integers(0, 4, (4, V))).astype(np.int32)
    c.o["repetition"], c.o["frequency"] = np.array([1.2, 0.6, 1.1, 1.3], np.float32), np.array([0.2, -0.4, 0.1, 0.0], np.float32)
    c.o["top_k"], c.o["top_p"] = np.array([50, 50, 0, 7], np.int32), np.array([0.9, 1.0, 0.8, 1.0], np.float32)
    c.o["min_p"][:] = 0
    _cut(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [float("nan"), float("inf")])
def test_a_value_that_is_no_number_far_behind_in_a_row_of_which_few_are_kept(odd, dtype):
    c = lg.Call(3, 0, 120000, dtype, ("k", "temp"), seed=32)
    c.o["top_k"] = np.array([20, 20, 20], np.int32)
    c.logits["target"][1, 0, 119000] = odd
    got = _cut(c)["target"]
    assert [(r > -float("inf")).sum().item() for r in got[[0, 2], 0]] == [20, 20] and (got[1, 0] > -float("inf")).sum().item() >= 119999


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_finite_values_of_masked_tokens(dtype):
    """The type's lowest number, or a large negative one, in place of -inf: top_k then reaches into them."""
    c = lg.Call(4, 0, 9001, dtype, ("k", "p"), seed=33)
    x = c.logits["target"]
    low = [torch.finfo(x.dtype).min, -1e9, -30000.0, -1e4]
    for b in range(4):
        x[b, 0, torch.arange(9001) % 300 != b] = low[b]
    c.o["top_k"], c.o["top_p"] = np.array([50, 20, 9000, 31], np.int32), np.array([1.0, 0.9, 1.0, 0.999], np.float32)
    _cut(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [100.0, 127.0, 128.0, 250.0, 256.0, 700.0, -130.0, -200.0, -260.0])
def test_cut_rows_far_from_zero(top, dtype):
    """As a low temperature makes them, on both sides of where the bins end."""
    c = lg.Call(3, 0, 5003, dtype, ("k", "p", "m"), seed=35)
    c.logits["target"].sub_(c.logits["target"].max(dim=-1, keepdim=True).values).mul_(4).add_(top)
    c.o["top_k"], c.o["top_p"], c.o["min_p"] = np.array([0, 30, 0], np.int32), np.array([0.9, 0.8, 1.0], np.float32), np.array([0, 0, 0.01], np.float32)
    _cut(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cut_rows_of_log_probabilities_with_a_sure_token(dtype):
    c = lg.Call(4, 0, 4001, dtype, ("k", "p"), seed=36)
    x = c.logits["target"]
    x.copy_(torch.log_softmax(x.double() + torch.where(torch.arange(4001) == 9, torch.tensor([8.0, 14.0, 22.0, 60.0]).view(4, 1, 1), 0.0), -1).to(x.dtype))
    c.o["top_k"], c.o["top_p"] = np.array([0, 5, 0, 0], np.int32), np.array([0.999, 0.99, 0.9, 0.5], np.float32)
    _cut(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_equal_values_at_the_cut_are_kept_by_rising_id(dtype):
    V = 9000
    c = lg.Call(6, 0, V, dtype, ("k", "p"), seed=23)
    c.logits["target"].copy_(torch.randint(0, 12, (6, 1, V), generator=torch.Generator().manual_seed(5)).float())
    c.o["top_k"] = np.array([1, 750, 751, 3000, 0, 8999], np.int32)
    c.o["top_p"] = np.array([1.0, 1.0, 0.5, 0.9, 0.25, 0.75], np.float32)
    _cut(c)


def test_equal_weights_and_a_share_that_ends_on_a_token():
    # 1000 equal tokens: their weights sum without rounding, and exactly half of them come in front of the border
    c = lg.Call(3, 0, 1000, "f32", ("p",), seed=24)
    c.logits["target"].fill_(2.5)
    c.o["top_p"] = np.array([0.5, 0.25, 0.001], np.float32)
    assert [(r > -1).sum().item() for r in _cut(c)["target"][:, 0]] == [500, 250, 2]     # float(0.001) is a little above 1 / 1000


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_a_distribution_are_not_cut(dtype):
    c = lg.Call(5, 0, 3000, dtype, ("k", "p", "m"), seed=25)
    c.o["top_k"][:], c.o["top_p"][:], c.o["min_p"][:] = 3, 0.5, 0.5
    x = c.logits["target"]
    x[0, 0, 2999], x[1, 0, 0], x[2, 0] = float("nan"), float("inf"), -float("inf")
    x[3, 0, :-1] = -float("inf")                            # one token left: it stays
    got = _cut(c)["target"]
    assert (got[0, 0] > -float("inf")).sum() == 2999 and (got[3, 0] > -float("inf")).sum() == 1


def test_shares_that_are_no_shares():
    c = lg.Call(6, 0, 2000, "f32", ("k", "p", "m"), seed=26)
    c.o["top_k"] = np.array([-5, 0, 2 ** 31 - 1, -2 ** 31, 0, 0], np.int32)
    c.o["top_p"] = np.array([np.nan, 2.0, np.inf, 1.0, -1.0, 1.0], np.float32)
    c.o["min_p"] = np.array([np.nan, -1.0, 0.0, -np.inf, 0.0, 7.0], np.float32)
    got = c.run()["target"]
    assert torch.equal(got[:4], c.logits["target"][:4])
    assert [(r > -float("inf")).sum().item() for r in got[4:, 0]] == [1, 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cut_rows_off_the_boundaries(dtype):
    for lead in ((1, 1), (5, 2), (0, 7)):
        c = lg.Call(4, 1, 2051, dtype, ("temp", "k", "p", "m"), seed=27)
        _cut(c, lead=lead)


def test_cut_tree_rows():
    c = lg.Call(2, 12, 3000, "bf16", ("pen", "mask", "temp", "k", "p", "m"), call="tree", seed=28)
    _cut(c)


# ---- token counts ---------------------------------------------------------------------------------
def _ragged(lists):
    flat = [t for x in lists for t in x]
    return lg.dev(np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)), lg.dev(np.array(flat or [0], np.int32))


def _state(B, V):
    room = torch.full((B * V + 64,), -77, dtype=torch.int32, device="cuda"), torch.full((B * ((V + 31) // 32) + 64,), -77, dtype=torch.int32, device="cuda")
    return room, room[0][:B * V].view(B, V), room[1][:B * ((V + 31) // 32)].view(B, -1)


def _same_state(room, counts, seen, want):
    assert np.array_equal(counts.cpu().numpy(), want[0]) and np.array_equal(seen.cpu().numpy().view(np.uint32), want[1])
    assert (room[0][counts.numel():] == -77).all() and (room[1][seen.numel():] == -77).all(), "stored behind the last sequence"


@pytest.mark.parametrize("V", [1, 31, 32, 33, 1000, 8192, 8193, 40001])
def test_history_from_ragged_prompts(V):
    rng = np.random.default_rng(V)
    lengths = [0, 1, 5, 3000, 0, 70000 if V == 40001 else 700]
    prompts = [rng.integers(-2, V + 2, n).tolist() for n in lengths]
    outputs = [rng.integers(-2, V + 2, n // 3).tolist() for n in reversed(lengths)]
    room, counts, seen = _state(6, V)
    (po, pt), (oo, ot) = _ragged(prompts), _ragged(outputs)
    s = torch.cuda.current_stream().cuda_stream
    assert fsd.fsd_history_build(po, pt, oo, ot, 6, V, counts, seen, s) == 0
    _same_state(room, counts, seen, lo.build(prompts, outputs, V))
    assert fsd.fsd_history_build(po, pt, None, None, 6, V, counts, seen, s) == 0
    _same_state(room, counts, seen, lo.build(prompts, [[]] * 6, V))


def test_history_of_one_token_many_times_and_of_offsets_that_fall():
    V, n = 500, 200000
    room, counts, seen = _state(2, V)
    tokens = lg.dev(np.full(n, 499, np.int32))
    assert fsd.fsd_history_build(lg.dev(np.array([0, n, 5], np.int32)), tokens, lg.dev(np.array([0, n, 5], np.int32)), tokens, 2, V, counts, seen,
                                 torch.cuda.current_stream().cuda_stream) == 0
    _same_state(room, counts, seen, lo.build([[499], []], [[499] * n, []], V))


@pytest.mark.parametrize("B,gamma,V", [(1, 1, 1), (5, 4, 33), (9, 40, 1000), (64, 8, 5000)])
def test_accepted_chain_tokens_join_the_history(B, gamma, V):
    rng = np.random.default_rng(B)
    tokens, n = rng.integers(-1, V + 1, (B, gamma)).astype(np.int32), rng.integers(-1, gamma + 3, B).astype(np.int32)
    nxt = rng.integers(-1, V, B).astype(np.int32)
    tokens[0] = tokens[0, 0]                               # the same token again and again
    before = lo.build([[int(t)] for t in rng.integers(0, V, B)], [[int(t)] * 3 for t in rng.integers(0, V, B)], V)
    room, counts, seen = _state(B, V)
    counts.copy_(lg.dev(before[0])); seen.copy_(lg.dev(before[1]))
    assert fsd.fsd_history_append_chain(lg.dev(tokens), lg.dev(n), lg.dev(nxt), B, gamma, V, counts, seen, torch.cuda.current_stream().cuda_stream) == 0
    _same_state(room, counts, seen, lo.append(*before, [[*tokens[b, :max(0, n[b])].tolist(), int(nxt[b])] for b in range(B)]))


def test_accepted_tree_tokens_join_the_history():
    B, N, V, width = 4, 7, 50, 3
    rng = np.random.default_rng(1)
    tokens = rng.integers(0, V, (B, N)).astype(np.int32)
    path = np.array([[0, 2, 5], [1, -1, -1], [0, 7, -9], [3, 4, 6]], np.int32)
    n, nxt = np.array([3, 1, 3, 0], np.int32), np.array([4, -1, 49, 50], np.int32)
    before = lo.build([[]] * B, [[]] * B, V)
    room, counts, seen = _state(B, V)
    counts.zero_(); seen.zero_()
    assert fsd.fsd_history_append_tree(lg.dev(tokens), lg.dev(path), lg.dev(n), lg.dev(nxt), B, N, width, V, counts, seen, torch.cuda.current_stream().cuda_stream) == 0
    _same_state(room, counts, seen, lo.append(*before, [[*[int(tokens[b, j]) for j in path[b, :n[b]] if 0 <= j < N], int(nxt[b])] for b in range(B)]))


# ---- as they are used: counts, processing, verification, counts ------------------------------------
@pytest.mark.parametrize("dtype,mode", [("f32", "sd"), ("bf16", "fsd"), ("bf16", "rfsd")])
def test_a_decoding_step(dtype, mode):
    B, gamma, V = 5, 4, 4096
    c = lg.Call(B, gamma, V, dtype, ("pen", "bias", "mask", "temp", "k", "p", "m"), seed=30)
    rng = np.random.default_rng(9)
    c.o["top_k"], c.o["top_p"] = np.array([0, 50, 0, 200, 0], np.int32), np.array([0.9, 1.0, 0.95, 0.8, 1.0], np.float32)
    c.o["min_p"] = np.array([0, 0, 0.01, 0, 0], np.float32)
    c.logits["draft"].copy_((c.logits["target"][:, :gamma].float() + 0.2 * torch.randn(B, gamma, V, generator=torch.Generator().manual_seed(3))).to(lg.TORCH[dtype]))
    prompts = [rng.integers(0, V, 30).tolist() for _ in range(B)]
    outputs = [rng.integers(0, V, 10).tolist() for _ in range(B)]
    s = torch.cuda.current_stream().cuda_stream
    room, counts, seen = _state(B, V)
    (po, pt), (oo, ot) = _ragged(prompts), _ragged(outputs)
    state = lo.build(prompts, outputs, V)
    c.o["counts"], c.o["seen"] = state
    u_accept, u_sample = rng.random((B, gamma)).astype(np.float32), rng.random(B).astype(np.float32)
    opts = fsd.make_opts(mode=mode, dtype=dtype, T=0.1)
    tokens, us, ua = lg.dev(c.tokens), lg.dev(u_sample), lg.dev(u_accept)
    n, nxt, st = (torch.full((B,), -7, dtype=torch.int32, device="cuda") for _ in range(3))
    D = torch.empty(B, gamma, device="cuda")
    wsb = fsd.fsd_workspace_bytes(B, gamma, V, opts)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    target, draft = c.logits["target"].cuda(), c.logits["draft"].cuda()
    process = c.opts(counts=counts, seen=seen)
    assert fsd.fsd_history_build(po, pt, oo, ot, B, V, counts, seen, s) == 0
    assert fsd.fsd_process_chain(target, draft, tokens, B, gamma, V, process, target, draft, s) == 0
    assert fsd.fsd_verify_chain(target, draft, tokens, ua, us, B, gamma, V, opts, n, nxt, D, st, ws, wsb, s) == 0
    assert fsd.fsd_history_append_chain(tokens, n, nxt, B, gamma, V, counts, seen, s) == 0
    torch.cuda.synchronize()
    got = {"target": target.cpu(), "draft": draft.cpu()}
    whole = c.run(c.opts(**CUT))
    c.check_values(whole)
    c.check_cut(got, whole)
    host = lambda x: x.view(torch.int16).numpy().view(np.uint16) if dtype == "bf16" else x.numpy()  # noqa: E731
    want = orc.verify_chain(host(got["target"]), host(got["draft"]), c.tokens, u_accept, u_sample, dtype=dtype, mode=mode, T=0.1)
    assert np.array_equal(n.cpu().numpy(), want.accept_len) and np.array_equal(nxt.cpu().numpy(), want.next_token)
    assert np.array_equal(st.cpu().numpy(), want.row_status)
    _same_state(room, counts, seen, lo.append(*state, [[*c.tokens[b, :want.accept_len[b]].tolist(), int(want.next_token[b])] for b in range(B)]))


def test_calls_in_a_graph_on_another_stream_and_two_at_once():
    c = lg.Call(4, 3, 20000, "bf16", ("pen", "bias", "mask", "temp", "k", "p", "m"), seed=31)
    want = c.run()
    opts, par = c.opts(), lg.dev(c.tokens)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ins = [{k: v.cuda() for k, v in c.logits.items()} for _ in range(2)]
    outs = [{k: torch.zeros_like(v) for k, v in x.items()} for x in ins]
    graphs = []
    torch.cuda.synchronize()
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[k]):
            assert fsd.fsd_process_chain(ins[k]["target"], ins[k]["draft"], par, c.B, c.P, c.V, opts, outs[k]["target"], outs[k]["draft"], streams[k].cuda_stream) == 0
        graphs.append(g)
    for _ in range(3):
        for x in outs:
            for v in x.values():
                v.zero_()
        torch.cuda.synchronize()
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                graphs[k].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x[s].cpu().view(torch.uint8), want[s].view(torch.uint8)) for x in outs for s in x)


def test_options_check_types_and_layouts_of_tensors():
    on = dict(device="cuda")
    for bad in (dict(top_k=torch.zeros(3, **on)), dict(top_p=torch.zeros(3, dtype=torch.float64, **on)), dict(counts=torch.zeros(4, 6, dtype=torch.int32, **on).t()),
                dict(top_p=torch.zeros(3))):
        with pytest.raises(ValueError):
            fsd.make_process_opts(**bad)


def test_an_error_that_an_earlier_call_left_behind_is_not_this_call_s():
    """The runtime keeps a thread's last error until somebody asks for it.  Here a copy from memory that is registered in part
    may leave one: the host-buffer call that wants the copy fails, the next call of another kind does not."""
    c = lg.Call(2, 1, 500, "bf16", ("pen", "temp"), seed=34)
    want = c.run()
    pages = torch.zeros(4 * 4096, dtype=torch.uint8)
    first = (pages.data_ptr() + 4095) // 4096 * 4096
    rt = torch.cuda.cudart()
    o = fsd.make_opts(dtype="bf16", T=0.1)
    n = fsd.fsd_host_staging_bytes(1, 1, 64, o)
    staging = torch.empty(n, dtype=torch.uint8, device="cuda")
    host = torch.zeros(4096, dtype=torch.uint8).pin_memory()
    at = [host.data_ptr() + 512 * k for k in range(8)]
    assert int(rt.cudaHostRegister(first, 4096, 0)) == 0
    try:
        rc = fsd.fsd_verify_chain_host(first + 4096 - 40, at[1], at[2], at[3], at[4], 1, 1, 64, o, at[5], at[6], at[7], at[7] + 64, staging, n,
                                       torch.cuda.current_stream().cuda_stream)
        assert rc in (0, -7)
        got = c.run()
    finally:
        assert int(rt.cudaHostUnregister(first)) == 0
    assert all(torch.equal(got[s].view(torch.uint8), want[s].view(torch.uint8)) for s in got)
