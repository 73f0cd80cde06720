"""Logit processing and token counts without a GPU: the argument checks of the calls, and pins of their oracle."""

import ctypes
import math

import numpy as np
import pytest

import paper_2502_20704_b200 as fsd
from oracle import fsd_logits_oracle as lo
from paper_2502_20704_b200 import binding, build


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


A = 1 << 20          # addresses that nothing is read from: every call below is refused on the host


def _chain(o="own", **kw):
    a = dict(t=A, d=A * 2, tok=A * 3, B=2, g=3, V=64, to=A * 4, do=A * 5)
    a.update(kw)
    o = fsd.make_process_opts(dtype="f32") if o == "own" else o
    return fsd.fsd_process_chain(a["t"], a["d"], a["tok"], a["B"], a["g"], a["V"], o, a["to"], a["do"], None)


def test_default_options():
    o = fsd.fsd_default_process_opts()
    assert o.struct_size == ctypes.sizeof(fsd.FsdProcessOpts) and o.logit_dtype == 1
    assert all(getattr(o, name) is None for name, _ in o._fields_[2:])


def test_chain_refusals():
    assert _chain(None) == binding.FSD_ERR_NULL
    assert _chain(t=None) == binding.FSD_ERR_NULL
    assert _chain(to=None) == binding.FSD_ERR_NULL
    assert _chain(d=None) == binding.FSD_ERR_NULL          # an output without its input
    assert _chain(do=None) == binding.FSD_ERR_NULL
    assert _chain(B=0) == binding.FSD_ERR_SHAPE
    assert _chain(g=-1) == binding.FSD_ERR_SHAPE
    assert _chain(V=0) == binding.FSD_ERR_SHAPE
    assert _chain(V=(1 << 30) + 1) == binding.FSD_ERR_SHAPE
    assert _chain(B=1 << 20, g=1 << 12) == binding.FSD_ERR_SHAPE
    for k in ("t", "to", "d", "do", "tok"):
        assert _chain(**{k: A * 9 + 2}) == binding.FSD_ERR_ALIGN, k
    # outputs over inputs that they are not the same as
    assert _chain(to=A + 4) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(to=A * 2) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(do=A * 4) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(do=A) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(to=A * 3 - 8) == binding.FSD_ERR_UNSUPPORTED
    o = fsd.make_process_opts(dtype="f32", counts=A * 6, seen=A * 7)
    assert _chain(o, to=A * 6) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(o, do=A * 7 - 4) == binding.FSD_ERR_UNSUPPORTED


def test_option_refusals():
    for field, value, code in (("struct_size", 8, binding.FSD_ERR_ENUM), ("logit_dtype", 2, binding.FSD_ERR_ENUM), ("logit_dtype", -1, binding.FSD_ERR_ENUM),
                               ("counts", A * 6, binding.FSD_ERR_NULL), ("seen", A * 6, binding.FSD_ERR_NULL), ("bias_tokens", A * 6, binding.FSD_ERR_NULL),
                               ("bias_values", A * 6, binding.FSD_ERR_NULL), ("bias_offsets", A * 6, binding.FSD_ERR_NULL)):
        o = fsd.make_process_opts(dtype="f32")
        setattr(o, field, value)
        assert _chain(o) == code, field
    for name, _ in fsd.FsdProcessOpts._fields_[2:]:
        o = fsd.make_process_opts(dtype="f32", counts=A * 6, seen=A * 6, bias_offsets=A * 6, bias_tokens=A * 6, bias_values=A * 6)
        setattr(o, name, A * 6 + 2)
        assert _chain(o) == binding.FSD_ERR_ALIGN, name
    with pytest.raises(TypeError):
        fsd.make_process_opts(top_q=None)
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        fsd.make_process_opts(top_k=torch.zeros(3))
    with pytest.raises(ValueError):
        fsd.make_process_opts(top_p=torch.zeros(3, dtype=torch.float64))
    with pytest.raises(ValueError):
        fsd.make_process_opts(counts=torch.zeros(4, 6, dtype=torch.int32).t())


def test_tree_refusals():
    o = fsd.make_process_opts(dtype="bf16")

    def tree(opts=o, t=A, d=A * 2, par=A * 3, tok=A * 6, N=5, to=A * 4, do=A * 5):
        return fsd.fsd_process_tree(t, d, par, tok, 2, N, 64, opts, to, do, None)

    assert tree(par=None) == binding.FSD_ERR_NULL
    assert tree(opts=None) == binding.FSD_ERR_NULL
    assert tree(N=0) == binding.FSD_ERR_SHAPE
    assert tree(N=1025) == binding.FSD_ERR_SHAPE
    assert tree(t=A + 1) == binding.FSD_ERR_ALIGN
    assert tree(par=A * 3 + 2) == binding.FSD_ERR_ALIGN
    assert tree(to=A * 3 - 8) == binding.FSD_ERR_UNSUPPORTED


def test_history_refusals():
    build_ = lambda po=A, pt=A, oo=A, ot=A, B=2, V=64, c=A, s=A: fsd.fsd_history_build(po, pt, oo, ot, B, V, c, s, None)  # noqa: E731
    for k in ("po", "pt", "c", "s", "oo", "ot"):
        assert build_(**{k: None}) == binding.FSD_ERR_NULL, k
        assert build_(**{k: A + 2}) == binding.FSD_ERR_ALIGN, k
    assert build_(B=0) == build_(V=0) == build_(V=(1 << 30) + 1) == build_(B=1 << 30, V=1 << 30) == binding.FSD_ERR_SHAPE
    chain = lambda d=A, n=A, x=A, B=2, g=3, V=64, c=A, s=A: fsd.fsd_history_append_chain(d, n, x, B, g, V, c, s, None)  # noqa: E731
    for k in ("d", "n", "x", "c", "s"):
        assert chain(**{k: None}) == binding.FSD_ERR_NULL, k
        assert chain(**{k: A + 1}) == binding.FSD_ERR_ALIGN, k
    assert chain(B=0) == chain(g=0) == chain(V=0) == chain(B=1 << 20, g=1 << 12) == binding.FSD_ERR_SHAPE
    tree = lambda d=A, p=A, n=A, x=A, N=3, w=2, V=64, c=A, s=A: fsd.fsd_history_append_tree(d, p, n, x, 2, N, w, V, c, s, None)  # noqa: E731
    for k in ("d", "p", "n", "x", "c", "s"):
        assert tree(**{k: None}) == binding.FSD_ERR_NULL, k
    assert tree(N=0) == tree(w=0) == tree(V=0) == binding.FSD_ERR_SHAPE


# ---- the oracle, by hand -----------------------------------------------------------------------
def test_oracle_process_by_hand():
    x = [2.0, -2.0, 1.0, 0.5]
    counts, seen = np.array([3, 0, 0, 0], np.int32), np.array([0b0011], np.uint32)
    y, _ = lo.process_row(x, counts, seen, drafted=[2, 2, 9, -1], repetition=2.0, frequency=0.25, presence=0.5, biases=[(3, 9.0), (3, 1.0), (7, 5.0)],
                          allowed=np.array([0b1101], np.uint32), temperature=0.5)
    # token 0: 2/2 - 0.75 - 0.5; token 1: masked; token 2, drafted twice: 1/2 - 0.5 - 0.5; token 3: the last bias
    assert y.tolist() == [-0.5, -math.inf, -1.0, 3.0]
    y, _ = lo.process_row(x, counts, seen, repetition=2.0)
    assert y.tolist() == [1.0, -4.0, 1.0, 0.5]


def test_oracle_contexts_by_hand():
    assert lo.context(None, 3) == [0, 1, 2]
    parent = [-1, 0, 0, 2, 7, 4]          # node 4's parent is not below it
    assert lo.context(parent, 0) == [] and lo.context(parent, 4) == [3, 2, 0] and lo.context(parent, 6) == [5, 4]
    assert lo.context_row(parent, "draft", 3) == 3 and lo.context_row(parent, "draft", 4) == 0 and lo.context_row(None, "draft", 2) == 2


def test_oracle_kept_by_hand():
    L = np.log
    y = L([0.1, 0.4, 0.2, 0.2, 0.1])
    of = lambda **kw: np.flatnonzero(lo.kept(y, **kw)).tolist()  # noqa: E731
    assert of(top_k=1) == [1] and of(top_k=2) == [1, 2] and of(top_k=3) == [1, 2, 3] and of(top_k=4) == [0, 1, 2, 3] and of(top_k=0) == of(top_k=5) == [0, 1, 2, 3, 4]
    assert of(top_p=0.3) == [1] and of(top_p=0.41) == [1, 2] and of(top_p=0.61) == [1, 2, 3] and of(top_p=0.0) == [1] and of(top_p=1.0) == [0, 1, 2, 3, 4]
    assert of(top_k=3, top_p=0.55) == [1, 2]                # 0.4 of the three's 0.8 is half
    assert of(top_k=3, top_p=0.45) == [1]
    assert of(min_p=0.49) == [1, 2, 3] and of(min_p=1.5) == [1] and of(min_p=0.0) == [0, 1, 2, 3, 4]
    assert lo.kept([-math.inf, -math.inf], top_k=1).all() and lo.kept([math.nan, 1.0], top_k=1).all() and lo.kept([math.inf, 1.0], top_k=1).all()
    assert lo.kept([0.0, -0.0, -math.inf], top_k=1).tolist() == [True, False, False]


def test_oracle_history_by_hand():
    counts, seen = lo.build([[1, 40, 99, -1], []], [[1, 1, 33], [0]], 41)
    assert counts[0].nonzero()[0].tolist() == [1, 33] and counts[0, 1] == 2 and counts[1].sum() == 1
    assert [int(w) for w in seen[0]] == [0b10, 1 << 8 | 1 << 1] and [int(w) for w in seen[1]] == [1, 0]
    c2, s2 = lo.append(counts, seen, [[1, -1, 2], [41]])
    assert c2[0, 1] == 3 and c2[0, 2] == 1 and int(s2[0, 0]) == 0b110 and np.array_equal(c2[1], counts[1])


# ---- calls that are refused have done nothing ------------------------------------------------------
def test_a_cut_that_cannot_be_launched_is_refused_in_front_of_the_first_kernel():
    """Biases and a cut are two kernels; fp32 rows by eight blocks each are more blocks than a launch may have.  (Where the first kernel
    went ahead this gave FSD_ERR_CUDA without a GPU.)"""
    far = 1 << 50
    o = fsd.make_process_opts(dtype="f32", bias_offsets=A, bias_tokens=A * 64, bias_values=A * 128, top_p=A * 192)
    assert _chain(o, t=far, d=far * 2, to=far * 3, do=far * 4, tok=None, B=1 << 20, g=128, V=140000) == binding.FSD_ERR_SHAPE


def test_an_output_that_is_another_input_of_the_same_address_is_refused():
    o = fsd.make_process_opts(dtype="f32", repetition=A, temperature=A * 2)
    plain = fsd.make_process_opts(dtype="f32")
    assert _chain(plain, t=A, to=A, d=A) == binding.FSD_ERR_UNSUPPORTED          # the draft's rows are read from what becomes the target's
    assert _chain(plain, t=A, d=A, do=A) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(plain, t=A, to=A, tok=A) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(plain, d=A * 2, do=A * 2, tok=A * 2) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(o, t=A, to=A) == binding.FSD_ERR_UNSUPPORTED
    assert _chain(o, d=A * 2, do=A * 2, t=A * 9) == binding.FSD_ERR_UNSUPPORTED
    tree = lambda t, d, par, to, do: fsd.fsd_process_tree(t, d, par, None, 2, 3, 64, plain, to, do, None)  # noqa: E731
    assert tree(A, A * 2, A, A, A * 5) == binding.FSD_ERR_UNSUPPORTED
    assert tree(A, A, A * 9, A, A * 5) == binding.FSD_ERR_UNSUPPORTED


def test_oracle_masks_hold_at_any_temperature():
    y, _ = lo.process_row([1.0, -math.inf, 2.0, -math.inf], allowed=np.array([0b0011], np.uint32), temperature=math.inf)
    assert y[0] == 0.0 and math.isnan(y[1]) and y[2:].tolist() == [-math.inf, -math.inf]
