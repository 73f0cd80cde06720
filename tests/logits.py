"""Helpers of the tests of logit processing: seeded calls with every option, run through the C ABI and by the oracle.

Tolerance of a processed value, derived from the arithmetic the header states: at most eight roundings to single precision
(1 / repetition, the product, frequency * n and its difference, presence, bias, 1 / temperature, the product), each at most half a
step of a value no larger than `size`, then one to the stored type."""

from __future__ import annotations

import numpy as np
import torch

import paper_2502_20704_b200 as fsd
from oracle import fsd_logits_oracle as lo

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
# half of the smallest step that a value near zero can be off by in storage (subnormals)
TINY = {"bf16": 2.0 ** -134, "f32": 2.0 ** -150}


def bits_of(may: np.ndarray) -> np.ndarray:
    """[..., V] truth values as [..., W] words."""
    V = may.shape[-1]
    W = (V + 31) // 32
    padded = np.zeros(may.shape[:-1] + (W * 32,), dtype=np.uint8)
    padded[..., :V] = may
    return np.packbits(padded, axis=-1, bitorder="little").view("<u4").reshape(may.shape[:-1] + (W,)).astype(np.uint32)


def dev(a):
    if a is None:
        return None
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).cuda()


def tree(rng, B, N):
    return np.array([[rng.integers(-1, j) if j else -1 for j in range(N)] for _ in range(B)], dtype=np.int32)


class Call:
    """A process call's inputs on the host.  Steps: any of pen, bias, mask, temp, k, p, m."""

    def __init__(self, B, P, V, dtype="bf16", steps=("pen", "bias", "mask", "temp"), call="chain", draft=True, seed=0, scale=3.0, hist=40):
        rng = np.random.default_rng([seed, B, P, V])
        self.B, self.P, self.V, self.dtype, self.call = B, P, V, dtype, call
        self.parent = tree(rng, B, P) if call == "tree" else None
        t = torch.from_numpy((rng.standard_normal((B, P + 1, V)) * scale).astype(np.float32)).to(TORCH[dtype])
        d = torch.from_numpy((rng.standard_normal((B, P, V)) * scale).astype(np.float32)).to(TORCH[dtype])
        self.logits = {"target": t, "draft": d if draft and P > 0 else None}
        # low ids often, so that tokens repeat; the history's, the drafted and the biased ones meet
        some = lambda *shape: np.minimum((rng.random(shape) ** 3 * V).astype(np.int32), V - 1)  # noqa: E731
        self.tokens = some(B, P) if P > 0 else None
        self.o = dict.fromkeys(("counts", "seen", "repetition", "frequency", "presence", "bias_offsets", "bias_tokens", "bias_values",
                                "allowed", "temperature", "top_k", "top_p", "min_p"))
        if "pen" in steps:
            n = [int(rng.integers(0, hist + 1)) for _ in range(B)]
            self.o["counts"], self.o["seen"] = lo.build([some(k).tolist() for k in n], [some(k // 2).tolist() for k in n], V)
            self.o["repetition"] = rng.choice([0.8, 1.0, 1.1, 1.5], B).astype(np.float32)
            self.o["frequency"] = rng.choice([-0.3, 0.0, 0.2, 0.7], B).astype(np.float32)
            self.o["presence"] = rng.choice([-0.5, 0.0, 0.4], B).astype(np.float32)
        if "bias" in steps:
            n = rng.integers(0, min(V, 20) + 1, B)
            self.o["bias_offsets"] = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
            total = max(1, int(n.sum()))
            self.o["bias_tokens"] = some(total)                                  # some more than once
            self.o["bias_values"] = (rng.standard_normal(total) * 2).astype(np.float32)
        if "mask" in steps:
            share = rng.choice([0.05, 0.5, 0.95, 1.0], (B, P + 1, 1))
            self.o["allowed"] = bits_of(rng.random((B, P + 1, V)) < share)
        if "temp" in steps:
            self.o["temperature"] = rng.choice([0.5, 0.7, 1.0, 1.3], B).astype(np.float32)
        if "k" in steps:
            self.o["top_k"] = rng.choice([-1, 0, 1, 2, 5, 50, V, V + 7, max(1, V // 2)], B).astype(np.int32)
        if "p" in steps:
            self.o["top_p"] = rng.choice([0.0, 0.1, 0.5, 0.9, 0.999, 1.0], B).astype(np.float32)
        if "m" in steps:
            self.o["min_p"] = rng.choice([0.0, 0.001, 0.1, 1.0], B).astype(np.float32)

    def opts(self, **instead):
        return fsd.make_process_opts(dtype=self.dtype, **{k: v if isinstance(v, torch.Tensor) else dev(v) for k, v in {**self.o, **instead}.items()})

    def run(self, opts=None, in_place=False, lead=(0, 0), stream=None, tokens="own"):
        """{side: processed rows}.  lead: elements that the inputs and the outputs start behind a 256-byte boundary."""
        opts = opts or self.opts()
        sides, outs, whole = {}, {}, []
        for side, x in self.logits.items():
            if x is None:
                sides[side] = outs[side] = None
                continue
            for which, lead_ in ((sides, lead[0]),) if in_place else ((sides, lead[0]), (outs, lead[1])):
                room = torch.full((x.numel() + 128 + lead_,), 7.0, dtype=x.dtype, device="cuda")
                which[side] = room[lead_:lead_ + x.numel()].view(x.shape)
                whole.append((room, lead_, x.numel()))
            sides[side].copy_(x)
            if in_place:
                outs[side] = sides[side]
        tok = dev(self.tokens) if isinstance(tokens, str) else tokens
        s = stream if stream is not None else torch.cuda.current_stream().cuda_stream
        if self.call == "tree":
            rc = fsd.fsd_process_tree(sides["target"], sides["draft"], dev(self.parent), tok, self.B, self.P, self.V, opts, outs["target"], outs["draft"], s)
        else:
            rc = fsd.fsd_process_chain(sides["target"], sides["draft"], tok, self.B, self.P, self.V, opts, outs["target"], outs["draft"], s)
        assert rc == 0, fsd.fsd_status_string(rc)
        torch.cuda.synchronize()
        for room, lead_, n in whole:
            assert (room[:lead_] == 7.0).all() and (room[lead_ + n:] == 7.0).all(), "stored outside the rows"
        if not in_place:
            for side, x in self.logits.items():
                assert x is None or torch.equal(sides[side].cpu().view(torch.uint8), x.view(torch.uint8)), "the input was written"
        return {side: None if v is None else v.cpu() for side, v in outs.items()}

    def want(self, side, b, r, tokens=True):
        """The oracle's row in double precision, and the magnitudes it went through."""
        row = lo.context_row(None if self.parent is None else self.parent[b], side, r)
        drafted = [int(self.tokens[b][j]) for j in lo.context(None if self.parent is None else self.parent[b], row)] if tokens and self.tokens is not None else []
        o, biases = self.o, ()
        if o["bias_offsets"] is not None:
            a, z = o["bias_offsets"][b], o["bias_offsets"][b + 1]
            biases = list(zip(o["bias_tokens"][a:z].tolist(), o["bias_values"][a:z].tolist()))
        at = lambda k: None if o[k] is None else o[k][b]  # noqa: E731
        return lo.process_row(self.logits[side][b, r].double().numpy(), counts=at("counts"), seen=at("seen"), drafted=drafted, repetition=at("repetition"),
                              frequency=at("frequency"), presence=at("presence"), biases=biases,
                              allowed=None if o["allowed"] is None else o["allowed"][b, row], temperature=at("temperature"))

    def check_values(self, got, tokens=True):
        for side, x in got.items():
            if x is None:
                continue
            for b in range(self.B):
                for r in range(x.shape[1]):
                    y = x[b, r].double().numpy()
                    want, size = self.want(side, b, r, tokens)
                    fin = np.isfinite(want)
                    assert np.array_equal(np.isnan(y), np.isnan(want)) and np.array_equal(y[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), (side, b, r)
                    off = np.abs(y[fin] - want[fin])
                    may = 8 * 2.0 ** -24 * size[fin] + HALF_STEP[self.dtype] * (np.abs(want[fin]) + 8 * 2.0 ** -24 * size[fin]) + TINY[self.dtype]
                    assert (off <= may).all(), (side, b, r, off.max(), np.flatnonzero(off > may)[:4])

    def check_cut(self, got, whole):
        """got: the rows as cut off; whole: the same call's without top_k, top_p and min_p.  What is kept is what the
        oracle keeps of the stored values, bit for bit."""
        at = lambda k, b: None if self.o[k] is None else self.o[k][b].item()  # noqa: E731
        for side, x in got.items():
            if x is None:
                continue
            for b in range(self.B):
                for r in range(x.shape[1]):
                    y = whole[side][b, r]
                    keep = lo.kept(y.double().numpy(), at("top_k", b), at("top_p", b), at("min_p", b))
                    want = torch.where(torch.from_numpy(keep), y, torch.tensor(-float("inf"), dtype=y.dtype))
                    same = (x[b, r] == want) | (x[b, r].isnan() & want.isnan())
                    assert same.all(), (side, b, r, at("top_k", b), at("top_p", b), at("min_p", b), torch.nonzero(~same)[:4].flatten().tolist(),
                                        int((x[b, r] > -float("inf")).sum()), int(keep.sum()))
