"""Logit processing and token counts by the debug build, whose kernels check their indices and ranges, in a process of its own:
results as the oracle's, and no check that failed."""

import os
import subprocess
import sys

import pytest

import paper_2502_20704_b200 as fsd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_SCRIPT = r"""
import numpy as np, torch
import paper_2502_20704_b200 as fsd
from oracle import fsd_logits_oracle as lo
from tests import logits as lg

assert fsd.fsd_debug_checks()[0], "this process must have loaded the debug build"
ALL = ("pen", "bias", "mask", "temp")
CUT = dict(top_k=None, top_p=None, min_p=None)

def none_failed(what):
    torch.cuda.synchronize()
    word = fsd.fsd_debug_process_word()
    assert word == 0, f"range check failed: bits {word:#x} ({what})"

def values(*a, lead=(0, 0), **kw):
    c = lg.Call(*a, **kw)
    c.check_values(c.run(lead=lead))
    none_failed(("values", a, kw, lead))

def cut(*a, lead=(0, 0), change=None, **kw):
    c = lg.Call(*a, **kw)
    if change:
        change(c)
    for in_place in (False, True):
        got = c.run(lead=(lead[0], lead[0]) if in_place else lead, in_place=in_place)
        none_failed(("cut", a, kw, lead, in_place))
        c.check_cut(got, c.run(c.opts(**CUT), lead=lead))
        none_failed(("whole", a, kw, lead, in_place))

for dtype in ("f32", "bf16"):
    for B, P, V in ((1, 0, 1), (2, 1, 7), (3, 2, 33), (2, 5, 4099), (2, 3, 8192)):
        for lead in ((0, 0), (3, 1), (0, 5)):
            values(B, P, V, dtype, lead=lead)
            cut(B, P, V, dtype, ALL + ("k", "p", "m"), lead=lead, seed=1)
            cut(B, P, V, dtype, ("pen", "mask", "temp", "k", "p", "m"), lead=lead, seed=2)
    values(2, 40, 1000, dtype, call="tree", seed=3)
    cut(2, 12, 3000, dtype, ("pen", "mask", "temp", "k", "p", "m"), call="tree", seed=4)

    def few(c):
        c.o["top_k"], c.o["top_p"] = np.array([50, 0, 3], np.int32), np.array([1.0, 0.9, 0.5], np.float32)
        c.o["min_p"][:] = 0
    for V in (32000, 50257, 100003, 300001, 800001):        # rows of one block and of eight, in two kernels, and off chip
        cut(3, 0, V, dtype, ("pen", "temp", "k", "p", "m"), change=few, seed=5, hist=3000)

    def full(c):                                            # more sparse ids than are listed
        rng = np.random.default_rng(7)
        used = rng.random((3, 60000)) < np.array([[1.0], [0.5], [0.01]])
        c.o["seen"], c.o["counts"] = lg.bits_of(used), (used * rng.integers(0, 4, (3, 60000))).astype(np.int32)
        few(c)
    cut(3, 2, 60000, dtype, ("pen", "temp", "k", "p", "m"), change=full, seed=6)

    def shape(x):
        def change(c):
            c.logits["target"].copy_(x.expand(3, 1, -1))
            few(c)
        return change
    n = torch.randn(3, 1, 20000, generator=torch.Generator().manual_seed(1))
    for x in (n * 0 - 3.25, n * 200 - 3000, n * 1e30, n * 1e-6, torch.where(n > 3, n, torch.tensor(-float("inf"))), torch.where(n > 0, n, torch.tensor(-30000.0))):
        cut(3, 0, 20000, dtype, ("k", "p", "m"), change=shape(x))

s = torch.cuda.current_stream().cuda_stream
rng = np.random.default_rng(2)
for V in (1, 33, 11264, 11265, 40001):
    prompts, outputs = [rng.integers(-2, V + 2, n).tolist() for n in (0, 700, 5000)], [rng.integers(-2, V + 2, n).tolist() for n in (100, 0, 3000)]
    def ragged(lists):
        flat = [t for x in lists for t in x]
        return lg.dev(np.concatenate([[0], np.cumsum([len(x) for x in lists])]).astype(np.int32)), lg.dev(np.array(flat, np.int32))
    counts, seen = torch.zeros(3, V, dtype=torch.int32, device="cuda"), torch.zeros(3, (V + 31) // 32, dtype=torch.int32, device="cuda")
    (po, pt), (oo, ot) = ragged(prompts), ragged(outputs)
    assert fsd.fsd_history_build(po, pt, oo, ot, 3, V, counts, seen, s) == 0
    none_failed(("history", V))
    want = lo.build(prompts, outputs, V)
    assert np.array_equal(counts.cpu().numpy(), want[0]) and np.array_equal(seen.cpu().numpy().view(np.uint32), want[1])
print("no check failed")
"""


@pytest.mark.gpu
def test_debug_build_finds_no_range_violation_in_logit_processing():
    from paper_2502_20704_b200 import build as lib_build
    lib = lib_build.build(debug=True)
    env = dict(os.environ, FSD_VERIFY_LIB=lib, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""))
    r = subprocess.run([sys.executable, "-c", _SCRIPT], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "no check failed" in r.stdout


def test_release_build_has_no_such_checks():
    from paper_2502_20704_b200 import build as lib_build
    lib_build.build()
    assert fsd.fsd_debug_process_word() == 0
