"""Performance cases of the operators around a verify call that shape logits: penalties for used tokens, biases, grammar
masks and temperature (``process``), the same with the distribution cut off by top-k, top-p and min-p (``truncate``), the
token counts these read, made from prompts (``build``) and moved on by what a verify call accepted (``append``).

``run`` computes a pass in elementary torch operations, or, where ``own`` is true, by the library's entry points.
Sizes are those of the verification cases: batches of 1 to 64, up to 15 drafted tokens or trees of up to 100 nodes,
vocabularies of 1000 to 256000 entries, whole multiples of 16 bytes a row and not, both logit types.
"""

from __future__ import annotations

import math
import random

import torch

own = False

ELEM = {"bf16": 2, "f32": 4}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
# most logits of one call (the largest listed case)
MOST = 64 * 17 * 152064


def _shape(kind, name, B, P, V, dtype="bf16", call="chain", draft=True, penalties=True, bias=0, mask=False, cut="", hist=2000):
    """P: drafted tokens a sequence (tree: nodes).  hist: tokens a sequence has behind it.  cut: which of top-k, top-p and
    min-p a batch's sequences use ("" none, "p" top-p alone, "kpm" a mixture, each sequence its own)."""
    return {"name": name, "kind": kind, "call": call, "B": B, "P": P, "V": V, "dtype": dtype, "draft": draft, "penalties": penalties,
            "bias": bias, "mask": mask, "cut": cut, "hist": hist}


def listed():
    return [
        # one interactive request that decodes token by token, no draft: launch and latency count
        _shape("process", "next_token_f32", 1, 0, 32000, dtype="f32", draft=False, hist=700),
        # a small serving batch: both models' rows, a caller's biases
        _shape("process", "small_batch", 16, 5, 32000, bias=300),
        # a vocabulary whose rows are not a multiple of 16 bytes, structured output, fp32
        _shape("process", "ragged_grammar_f32", 7, 3, 50257, dtype="f32", bias=40, mask=True),
        # structured output on a 128k vocabulary: a mask for every drafted position
        _shape("process", "grammar_128k", 32, 6, 128256, mask=True, bias=16),
        # tree drafting: each node's history is its ancestors
        _shape("process", "tree_60", 8, 60, 32000, call="tree", mask=True),
        # a full batch of long conversations on a 152k vocabulary
        _shape("process", "full_batch_152k", 64, 8, 152064, hist=16000),
        # sampling one token at a time from a cut distribution
        _shape("truncate", "sample_next_f32", 1, 0, 32000, dtype="f32", draft=False, cut="kpm", hist=700),
        # a small batch under top-p, both models' rows
        _shape("truncate", "sample_small_p", 16, 5, 32000, cut="p"),
        # a full batch, each sequence with settings of its own
        _shape("truncate", "sample_152k", 64, 8, 152064, cut="kpm"),
        # the counts of a batch of long prompts, as after a prefill or a resumed batch
        {"name": "prompts_128k", "kind": "build", "B": 32, "V": 128256, "hist": 32768},
        # what a chain call accepted joins the counts
        {"name": "accepted_chain", "kind": "append", "call": "chain", "B": 64, "P": 8, "V": 152064, "hist": 2000},
        # what a tree call accepted
        {"name": "accepted_tree", "kind": "append", "call": "tree", "B": 8, "P": 60, "V": 32000, "hist": 2000},
    ]


def _log_uniform(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def draw(rng):
    kind = rng.choice(["process", "process", "process", "truncate", "truncate", "truncate", "build", "append"])
    V = int(_log_uniform(rng, 1000, 256000))
    if rng.random() < 0.5:
        V -= V % 64
    B = int(round(_log_uniform(rng, 1, 64)))
    hist = int(_log_uniform(rng, 16, 32768))
    call = "tree" if rng.random() < 0.2 else "chain"
    P = rng.randint(4, 100) if call == "tree" else rng.randint(0, 15)
    if kind == "build":
        return {"kind": kind, "B": B, "V": V, "hist": hist}
    if kind == "append":
        return {"kind": kind, "call": call, "B": B, "P": max(P, 1), "V": V, "hist": hist}
    while B > 1 and B * (2 * P + 1) * V > MOST:
        B = B * 3 // 4
    c = _shape(kind, "", B, P, V, dtype=rng.choice(["bf16", "bf16", "f32"]), call=call, draft=P > 0 and rng.random() < 0.8,
               penalties=rng.random() < 0.8, bias=rng.choice([0, 0, 5, 300]), mask=rng.random() < 0.4,
               cut=rng.choice(["p", "kpm"]) if kind == "truncate" else "", hist=hist)
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _rows(g, n, V):
    """Logit rows of n contexts: small vocabularies 3 N(0, 1) with one spike of 8, large ones Zipf-shaped."""
    noise = torch.randn(n, V, generator=g, device="cuda")
    if V < 60000:
        noise.mul_(3.0)
        at = torch.randint(V, (n, 1), generator=g, device="cuda")
        return noise.scatter_add_(1, at, torch.full((n, 1), 8.0, device="cuda"))
    rank = torch.rand(n, V, generator=g, device="cuda").mul_(V).floor_().add_(1.0)
    return noise.mul_(0.5).add_(rank.log_(), alpha=-1.1)


def _tokens(g, shape, V):
    """Token ids as texts have them: low ids far more often than high ones."""
    return torch.rand(shape, generator=g, device="cuda").pow_(3.0).mul_(V).long().clamp_(max=V - 1)


def _pick(g, B, values):
    v = torch.tensor(values, dtype=torch.float32, device="cuda")
    return v[torch.randint(len(values), (B,), generator=g, device="cuda")]


def _parents(seed, B, N):
    """Draft trees of depth at most 6, four children a node at most."""
    rng, out = random.Random(int(seed) * 7919 + 11), []
    for _ in range(B):
        par, depth, kids = [], [], [0] * (N + 1)
        for j in range(N):
            can = [i for i in range(-1, j) if kids[i + 1] < 4 and (i < 0 or depth[i] < 6)]
            p = rng.choice(can) if can else -1
            par.append(p)
            depth.append(1 if p < 0 else depth[p] + 1)
            kids[p + 1] += 1
        out.append(par)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _pack(bits):
    """[..., V] truth values to [..., ceil(V / 32)] words."""
    V = bits.shape[-1]
    W = (V + 31) // 32
    bits = torch.nn.functional.pad(bits.to(torch.uint8), (0, W * 32 - V)).view(*bits.shape[:-1], W, 32)
    words = (bits.long() << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _history(g, B, V, n):
    """counts and seen of B sequences of n tokens, half of them a prompt's."""
    prompt, out = _tokens(g, (B, n - n // 2), V), _tokens(g, (B, n // 2), V)
    counts = torch.zeros(B, V, dtype=torch.int32, device="cuda")
    counts.scatter_add_(1, out, torch.ones_like(out, dtype=torch.int32))
    seen = counts > 0
    seen.scatter_(1, prompt, torch.ones_like(prompt, dtype=torch.bool))
    return counts, _pack(seen)


def _prepare_build(case, g):
    B, V, most = case["B"], case["V"], case["hist"]
    s = {"stream": torch.cuda.current_stream().cuda_stream}
    for name, top in (("prompt", most), ("output", max(1, most // 4))):
        # lengths spread over their logarithm, some sequences with nothing generated yet
        n = torch.rand(B, generator=g, device="cuda").mul_(math.log(top + 1)).exp_().long()
        n = torch.where(torch.rand(B, generator=g, device="cuda") < (0.3 if name == "output" else 0.0), 0, n)
        offsets = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        offsets[1:] = n.cumsum(0)
        s[name + "_offsets"], s[name + "_tokens"] = offsets, _tokens(g, (int(offsets[-1]) or 1,), V).to(torch.int32)
    s["counts"] = torch.empty(B, V, dtype=torch.int32, device="cuda")
    s["seen"] = torch.empty(B, (V + 31) // 32, dtype=torch.int32, device="cuda")
    return s


def _prepare_append(case, g, seed):
    B, P, V = case["B"], case["P"], case["V"]
    counts, seen = _history(g, B, V, case["hist"])
    s = {"counts": counts, "seen": seen, "tokens": _tokens(g, (B, P), V).to(torch.int32), "path": None,
         "next_token": _tokens(g, (B,), V).to(torch.int32), "stream": torch.cuda.current_stream().cuda_stream}
    if case["call"] == "tree":
        s["path"] = torch.full((B, 6), -1, dtype=torch.int32, device="cuda")
        parent = _parents(seed, B, P).tolist()
        depth = []
        for b in range(B):
            way, j = [], P - 1 - b % P
            while j >= 0:
                way.append(j)
                j = parent[b][j]
            s["path"][b, : len(way)] = torch.tensor(way[::-1], dtype=torch.int32)
            depth.append(len(way))
        s["accept_len"] = torch.tensor(depth, dtype=torch.int32, device="cuda")
    else:
        s["accept_len"] = torch.randint(P + 1, (B,), generator=g, device="cuda").to(torch.int32)
    return s


def prepare(case, seed):
    g = _generator(seed)
    if case["kind"] == "build":
        return {"case": case, **_prepare_build(case, g)}
    if case["kind"] == "append":
        return {"case": case, **_prepare_append(case, g, seed)}
    B, P, V, dt = case["B"], case["P"], case["V"], TORCH[case["dtype"]]
    tree = case["call"] == "tree"
    parent = _parents(seed, B, P) if tree else None
    target = torch.empty(B, P + 1, V, dtype=dt, device="cuda")
    draft = torch.empty(B, P, V, dtype=dt, device="cuda") if case["draft"] else None
    allowed = torch.empty(B, P + 1, (V + 31) // 32, dtype=torch.int32, device="cuda") if case["mask"] else None
    for b in range(B):
        rows = _rows(g, P + 1, V)
        target[b] = rows
        if draft is not None:
            base = rows[parent[b].long() + 1] if tree else rows[:P]
            draft[b] = base + 0.7 * torch.randn(P, V, generator=g, device="cuda")
        if allowed is not None:
            # inside a string a grammar allows nearly all, between its fields next to nothing; the end token always
            share = torch.where(torch.rand(P + 1, 1, generator=g, device="cuda") < 0.5, 0.02, 0.97)
            may = torch.rand(P + 1, V, generator=g, device="cuda") < share
            may[:, 0] = True
            allowed[b] = _pack(may)
    s = {"case": case, "target": target, "draft": draft, "allowed": allowed, "parent": parent,
         "tokens": _tokens(g, (B, P), V).to(torch.int32), "temperature": _pick(g, B, [0.6, 0.7, 0.8, 1.0, 1.2]),
         "target_out": torch.empty_like(target), "draft_out": torch.empty_like(draft) if draft is not None else None,
         "stream": torch.cuda.current_stream().cuda_stream}
    for k in ("counts", "seen", "repetition", "frequency", "presence", "bias_offsets", "bias_tokens", "bias_values", "top_k", "top_p", "min_p"):
        s[k] = None
    if case["penalties"]:
        s["counts"], s["seen"] = _history(g, B, V, case["hist"])
        s["repetition"] = _pick(g, B, [1.0, 1.05, 1.1, 1.3])
        s["frequency"], s["presence"] = _pick(g, B, [0.0, 0.2, 0.5]), _pick(g, B, [0.0, 0.4])
    if case["bias"]:
        n = min(case["bias"], V)
        at = (torch.arange(n, device="cuda") + torch.rand(B, n, generator=g, device="cuda") * 0.999) * (V / n)
        s["bias_tokens"] = at.long().clamp_(max=V - 1).to(torch.int32).view(-1)
        s["bias_values"] = torch.randn(B * n, generator=g, device="cuda").mul_(3.0)
        s["bias_offsets"] = torch.arange(B + 1, dtype=torch.int32, device="cuda") * n
    if "k" in case["cut"]:
        s["top_k"] = _pick(g, B, [0, 0, 20, 50, 200]).to(torch.int32)
    if "p" in case["cut"]:
        s["top_p"] = _pick(g, B, [0.8, 0.9, 0.95, 0.99] if case["cut"] == "p" else [1.0, 0.8, 0.9, 0.95])
    if "m" in case["cut"]:
        s["min_p"] = _pick(g, B, [0.0, 0.0, 0.02, 0.05])
    return s


# ---- the plain forms -------------------------------------------------------------------------
def _bits(words, V):
    """[..., W] words to [..., V] truth values."""
    return ((words.unsqueeze(-1) >> torch.arange(32, device=words.device)) & 1).bool().flatten(-2)[..., :V]


def _context(s, P):
    """[B, P + 1, P]: whether drafted token j stands before target row r (chain: j < r; tree: node r - 1 and its ancestors)."""
    dev = s["tokens"].device
    if s["parent"] is None:
        return (torch.arange(P, device=dev) < torch.arange(P + 1, device=dev).unsqueeze(1)).expand(s["tokens"].shape[0], P + 1, P)
    up = torch.nn.functional.one_hot(s["parent"].long() + 1, P + 1)[..., 1:].double()      # node j's parent, none for the root's children
    reach = torch.linalg.matrix_power(torch.eye(P, device=dev, dtype=torch.float64) + up, P) > 0.5
    return torch.cat([torch.zeros_like(reach[:, :1]), reach], dim=1)


def _plain_rows(s, x, before, allowed):
    """x [B, R, V] logits, before [B, R, P] the drafted tokens that stand before a row, allowed [B, R, W] or None."""
    B, R, V = x.shape
    P, out = before.shape[2], x.dtype
    x = x.float()
    col = lambda t: t.view(B, 1, 1)  # noqa: E731
    if s["counts"] is not None:
        n = s["counts"].unsqueeze(1).repeat(1, R, 1)
        n.scatter_add_(2, s["tokens"].long().unsqueeze(1).expand(B, R, P), before.to(torch.int32))
        used = _bits(s["seen"], V).unsqueeze(1) | (n > 0)
        x = torch.where(used, torch.where(x > 0, x * col(1.0 / s["repetition"]), x * col(s["repetition"])), x)
        x = x - col(s["frequency"]) * n
        x = x - torch.where(n > 0, col(s["presence"]), 0.0)
    if s["bias_offsets"] is not None:
        bias = torch.zeros(B, V, device=x.device)
        of = torch.searchsorted(s["bias_offsets"], torch.arange(s["bias_tokens"].numel(), device=x.device), right=True) - 1
        bias.view(-1).index_add_(0, of * V + s["bias_tokens"].long(), s["bias_values"])
        x = x + bias.unsqueeze(1)
    if allowed is not None:
        x = torch.where(_bits(allowed, V), x, -math.inf)
    x = (x * col(1.0 / s["temperature"])).to(out)
    if s["top_p"] is None:
        return x
    v, at = torch.sort(x.float(), dim=-1, descending=True, stable=True)
    place = torch.arange(V, device=x.device)
    first = v[..., :1].double()
    w = (v.double() - first).exp()
    if s["top_k"] is not None:
        k = torch.where((s["top_k"] <= 0) | (s["top_k"] >= V), V, s["top_k"])
        inside = place < col(k)
        w = torch.where(inside, w, 0.0)
    else:
        inside = (place >= 0).expand_as(w)
    below = w.cumsum(-1) - w
    keep = inside & ((below < col(s["top_p"].double()) * w.sum(-1, keepdim=True)) | col(s["top_p"] >= 1.0) | (place == 0))
    if s["min_p"] is not None:
        keep &= (v.double() - first >= col(s["min_p"].double()).log()) | col(s["min_p"] <= 0.0)
    kept = torch.where(keep, v, -math.inf).to(out)
    return torch.empty_like(x).scatter_(2, at, kept)


def _plain_process(s):
    P = s["case"]["P"]
    before = _context(s, P)
    got = {"target": _plain_rows(s, s["target"], before, s["allowed"])}
    if s["draft"] is not None:
        B = s["target"].shape[0]
        if s["parent"] is None:
            got["draft"] = _plain_rows(s, s["draft"], before[:, :P], None if s["allowed"] is None else s["allowed"][:, :P])
        else:       # node j was proposed after its parent, whose target row is parent + 1
            row = s["parent"].long() + 1
            b = torch.arange(B, device=row.device).unsqueeze(1)
            got["draft"] = _plain_rows(s, s["draft"], before[b, row], None if s["allowed"] is None else s["allowed"][b, row])
    return got


def _plain_build(s):
    B, V = s["case"]["B"], s["case"]["V"]

    def places(name):
        tokens, offsets = s[name + "_tokens"], s[name + "_offsets"]
        of = torch.searchsorted(offsets, torch.arange(tokens.numel(), device=tokens.device), right=True) - 1
        real = of < B
        return torch.where(real, of * V + tokens.long(), 0), real

    at, real = places("output")
    counts = torch.zeros(B * V, dtype=torch.int32, device=at.device).index_add_(0, at, real.to(torch.int32))
    at, real = places("prompt")
    seen = torch.zeros(B * V, dtype=torch.int32, device=at.device).index_add_(0, at, real.to(torch.int32))
    return {"counts": counts.view(B, V), "seen": _pack(((seen > 0) | (counts > 0)).view(B, V))}


def _plain_append(s):
    B, V = s["counts"].shape
    tokens = s["tokens"].long()
    if s["path"] is not None:
        tokens = tokens.gather(1, s["path"].long().clamp(min=0))
    real = torch.arange(tokens.shape[1], device=tokens.device) < s["accept_len"].unsqueeze(1)
    tokens = torch.cat([tokens, s["next_token"].long().unsqueeze(1)], dim=1)
    real = torch.cat([real, (s["next_token"] >= 0).unsqueeze(1)], dim=1)
    new = torch.zeros(B, V, dtype=torch.int32, device=tokens.device)
    new.scatter_add_(1, tokens.clamp(min=0), real.to(torch.int32))
    s["counts"].add_(new)
    s["seen"].bitwise_or_(_pack(new > 0))
    return {"counts": s["counts"], "seen": s["seen"]}


# ---- the library's calls ---------------------------------------------------------------------
def _ok(fsd, rc):
    if rc != 0:
        raise RuntimeError(fsd.fsd_status_string(rc))


def _own(s):
    import paper_2502_20704_b200 as fsd

    case = s["case"]
    if case["kind"] == "build":
        _ok(fsd, fsd.fsd_history_build(s["prompt_offsets"], s["prompt_tokens"], s["output_offsets"], s["output_tokens"], case["B"], case["V"],
                                       s["counts"], s["seen"], s["stream"]))
        return {"counts": s["counts"], "seen": s["seen"]}
    B, P, V = case["B"], case["P"], case["V"]
    if case["kind"] == "append":
        if case["call"] == "tree":
            _ok(fsd, fsd.fsd_history_append_tree(s["tokens"], s["path"], s["accept_len"], s["next_token"], B, P, s["path"].shape[1], V,
                                                 s["counts"], s["seen"], s["stream"]))
        else:
            _ok(fsd, fsd.fsd_history_append_chain(s["tokens"], s["accept_len"], s["next_token"], B, P, V, s["counts"], s["seen"], s["stream"]))
        return {"counts": s["counts"], "seen": s["seen"]}
    if "opts" not in s:         # a program makes the options once, with the buffers they point to
        arrays = {k: s[k] for k in ("counts", "seen", "repetition", "frequency", "presence", "bias_offsets", "bias_tokens", "bias_values", "allowed",
                                    "temperature", "top_k", "top_p", "min_p")}
        if s["bias_offsets"] is not None:       # of a token listed twice the call takes the last entry: both say what they add up to
            at = s["bias_tokens"].view(B, -1).long()
            arrays["bias_values"] = torch.zeros(B, V, device=at.device).scatter_add_(1, at, s["bias_values"].view(B, -1)).gather(1, at).view(-1)
        s["opts"] = fsd.make_process_opts(dtype=case["dtype"], **arrays)
    if case["call"] == "tree":
        _ok(fsd, fsd.fsd_process_tree(s["target"], s["draft"], s["parent"], s["tokens"], B, P, V, s["opts"], s["target_out"], s["draft_out"],
                                      s["stream"]))
    else:
        _ok(fsd, fsd.fsd_process_chain(s["target"], s["draft"], s["tokens"], B, P, V, s["opts"], s["target_out"], s["draft_out"], s["stream"]))
    return {"target": s["target_out"], **({"draft": s["draft_out"]} if s["draft"] is not None else {})}


def run(s):
    if own:
        return _own(s)
    kind = s["case"]["kind"]
    return _plain_build(s) if kind == "build" else _plain_append(s) if kind == "append" else _plain_process(s)


# ---- what a pass cannot do without -----------------------------------------------------------
def work(case):
    B, V = case["B"], case["V"]
    W = (V + 31) // 32
    if case["kind"] == "build":
        # lengths spread over their logarithm: top / ln(top) tokens on the average
        tokens = B * sum(top / math.log(top + 1) for top in (case["hist"], max(1, case["hist"] // 4)))
        return {"bytes": 4.0 * (tokens + B * V + B * W), "flops": tokens}
    P = case["P"]
    if case["kind"] == "append":
        # half the drafted tokens (tree: half of the depth of 6), the drawn one, their counts and bits there and back
        tokens = B * (1 + (3 if case["call"] == "tree" else P / 2))
        return {"bytes": 20.0 * tokens + 8.0 * B, "flops": tokens}
    rows = B * (P + 1 + (P if case["draft"] else 0))
    size = 2.0 * ELEM[case["dtype"]] * rows * V + (4.0 * B * (P + 1) * W if case["mask"] else 0.0)
    if case["penalties"]:
        size += 4.0 * B * (W + min(V, case["hist"] // 2))
    # a logit: a comparison, five products and sums; cut off, an exponential (its polynomial of eight) and two comparisons too
    return {"bytes": size + 8.0 * B * case["bias"] + 4.0 * B * P, "flops": (16.0 if case["cut"] else 6.0) * rows * V}


# ---- the definition in 64 bits, a row at a time ----------------------------------------------
def exact(case, seed):
    if case["kind"] in ("build", "append"):
        return None         # whole numbers
    s = prepare(case, seed)
    B, P, V, dt = case["B"], case["P"], case["V"], TORCH[case["dtype"]]
    inf, dev = math.inf, s["target"].device
    on_host = {k: s[k].tolist() for k in ("tokens", "parent", "bias_offsets", "repetition", "frequency", "presence", "temperature", "top_k", "top_p", "min_p")
               if s[k] is not None}
    wanted = {"target": torch.empty(B, P + 1, V, dtype=torch.float64, device=dev)}
    if s["draft"] is not None:
        wanted["draft"] = torch.empty(B, P, V, dtype=torch.float64, device=dev)
    bit = torch.arange(32, dtype=torch.int32, device=dev)
    for b in range(B):
        inv = None
        if s["seen"] is not None:
            base = s["counts"][b].double()
            inv = torch.bitwise_and(s["seen"][b].view(-1, 1), torch.bitwise_left_shift(torch.ones_like(bit), bit)).ne(0).view(-1)[:V]
        for name in wanted:
            for r in range(wanted[name].shape[1]):
                # the target row of the same context, and the drafted tokens before it
                row = r if name == "target" or s["parent"] is None else on_host["parent"][b][r] + 1
                if s["parent"] is None:
                    drafted = list(range(row))
                else:
                    drafted, j = [], row - 1
                    while j >= 0:
                        drafted.append(j)
                        j = on_host["parent"][b][j]
                x = s[name][b, r].double()
                if inv is not None:
                    n, used = base.clone(), inv.clone()
                    for j in drafted:
                        n[on_host["tokens"][b][j]] += 1
                        used[on_host["tokens"][b][j]] = True
                    rep = on_host["repetition"][b]
                    x[used & (x > 0)] /= rep
                    x[used & (s[name][b, r] <= 0)] *= rep
                    x -= on_host["frequency"][b] * n + on_host["presence"][b] * n.gt(0)
                if s["bias_offsets"] is not None:
                    lo, hi = on_host["bias_offsets"][b], on_host["bias_offsets"][b + 1]
                    x.index_put_((s["bias_tokens"][lo:hi].long(),), s["bias_values"][lo:hi].double(), accumulate=True)
                if s["allowed"] is not None:
                    words = s["allowed"][b, row].view(-1, 1)
                    x[torch.bitwise_and(words, torch.bitwise_left_shift(torch.ones_like(bit), bit)).eq(0).view(-1)[:V]] = -inf
                x /= on_host["temperature"][b]
                if case["cut"]:
                    y = x.to(dt).double()       # the cut goes by the values as they are stored
                    order = torch.argsort(-y, stable=True)
                    k = on_host["top_k"][b] if s["top_k"] is not None else 0
                    order = order[: k if 0 < k < V else V]
                    p = torch.softmax(y[order], 0)
                    if on_host["top_p"][b] < 1:
                        order = order[: max(1, int((p.cumsum(0) - p < on_host["top_p"][b]).sum()))]
                    if s["min_p"] is not None and on_host["min_p"][b] > 0:
                        order = order[y[order] - y[order[0]] >= math.log(on_host["min_p"][b])]
                    out = torch.full_like(x, -inf)
                    out[order] = x[order]
                    x = out
                wanted[name][b, r] = x
    return wanted
