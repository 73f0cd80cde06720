"""The first call of a process that cuts rows off puts a table on the device.  Each test is a process of its own."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu

_PRELUDE = r"""
import numpy as np, torch
import paper_2502_20704_b200 as fsd
from tests import logits as lg

CUT = {"top_k": None, "top_p": None, "min_p": None}
c = lg.Call(4, 2, 5000, DTYPE, STEPS, seed=50)
if c.o["top_p"] is not None:
    c.o["top_p"] = np.array([0.9, 0.99, 0.5, 0.95], np.float32)
side = torch.cuda.Stream()                                  # (does not wait for the default stream, nor that for it)
ins = {k: v.cuda() for k, v in c.logits.items()}
tok, opts = lg.dev(c.tokens), c.opts()

def call(outs, stream):
    rc = fsd.fsd_process_chain(ins["target"], ins["draft"], tok, c.B, c.P, c.V, opts, outs["target"], outs["draft"], stream)
    assert rc == 0, fsd.fsd_status_string(rc)
"""

# the default stream has much to do when the call is made
_BUSY = _PRELUDE + r"""
whole = c.run(c.opts(**CUT))                                # (CUDA has loaded the library's kernels with it, where it loads all at once)
outs = {k: torch.zeros_like(v) for k, v in ins.items()}
done = torch.cuda.Event()
torch.cuda.synchronize()
torch.cuda._sleep(2_000_000_000)                            # about a second
done.record()
call(outs, side.cuda_stream)
side.synchronize()
print("the default stream is done:", done.query())
c.check_cut({k: v.cpu() for k, v in outs.items()}, whole)
"""

# two threads, each on a stream of its own
_THREADS = _PRELUDE + r"""
import threading
outs = [{k: torch.zeros_like(v) for k, v in ins.items()} for _ in range(4)]
streams = [torch.cuda.Stream() for _ in outs]
torch.cuda.synchronize()
gate = threading.Barrier(len(outs))
failed = []

def one(k):
    try:
        gate.wait()
        call(outs[k], streams[k].cuda_stream)
    except BaseException as e:
        failed.append(e)

threads = [threading.Thread(target=one, args=(k,)) for k in range(len(outs))]
[t.start() for t in threads]
[t.join() for t in threads]
assert not failed, failed
torch.cuda.synchronize()
whole = c.run(c.opts(**CUT))
for x in outs:
    c.check_cut({k: v.cpu() for k, v in x.items()}, whole)
"""

# while another stream's work is being captured
_BESIDE_A_CAPTURE = _PRELUDE + r"""
outs = {k: torch.zeros_like(v) for k, v in ins.items()}
x = torch.zeros(100, device="cuda")
g = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g, stream=torch.cuda.Stream(), capture_error_mode="global"):
    x += 1
    call(outs, side.cuda_stream)
    x += 1
side.synchronize()
x.zero_()
g.replay()
assert (x == 2).all()
c.check_cut({k: v.cpu() for k, v in outs.items()}, c.run(c.opts(**CUT)))
"""


def _run(script, dtype, steps, **env):
    script = script.replace("DTYPE", repr(dtype)).replace("STEPS", repr(steps))
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, env=dict(os.environ, PYTHONPATH=ROOT + os.pathsep + os.environ.get("PYTHONPATH", ""), **env),
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    return r.stdout


@pytest.mark.parametrize("loading", ["LAZY", "EAGER"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_first_call_beside_a_busy_default_stream(dtype, loading):
    out = _run(_BUSY, dtype, ("pen", "temp", "p"), CUDA_MODULE_LOADING=loading)
    # (CUDA waits for the device when it loads a kernel at its first use; the call itself does not)
    assert loading == "LAZY" or "the default stream is done: False" in out, "the call waited for the default stream"


def test_first_calls_of_several_threads():
    _run(_THREADS, "bf16", ("temp", "p"))


def test_a_first_call_while_another_stream_is_captured():
    _run(_BESIDE_A_CAPTURE, "bf16", ("temp", "p"))
