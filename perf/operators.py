"""Performance cases of the operators on fixed vocabularies: rows by token, their gradient, rows in 4 bits and scores against them.

Four kinds of pass:

  rows         out[i] = scale * weight[token i]: the input layer of a sequence model
  grad         its gradient, grad_weight[v] = scale * sum of grad_out[i] over the tokens i that are v, either the whole of it or
               added to a buffer that holds the steps before
  packed_rows  rows looked up in a matrix held in 4 bits with one scale for each group of columns (value = (q - 8) * scale, two
               columns in a byte, the even one in the low half)
  scores       out[m, v] = <x[m], row v> for every row of such a matrix: candidate retrieval, or an output layer

Tokens are Zipf ranks in an order of their own, a share of them padding, which looks up as zeros and has no gradient.
"""
import functools
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
PADDING = 0
MOST_BYTES = 1.0e9       # of a drawn case
MOST_FLOPS = 8.0e9


def _rows(name, n, vocab, dim, w, o, scaled=True, pad=0.02, zipf=1.05, tokens="i64"):
    return {"name": name, "kind": "rows", "n": n, "vocab": vocab, "dim": dim, "in": w, "out": o, "scaled": scaled, "pad": pad,
            "zipf": zipf, "tokens": tokens}


def _grad(name, n, vocab, dim, g, o, add, scaled=True, pad=0.05, zipf=1.05, tokens="i64"):
    return {"name": name, "kind": "grad", "n": n, "vocab": vocab, "dim": dim, "in": g, "out": o, "add": add, "scaled": scaled,
            "pad": pad, "zipf": zipf, "tokens": tokens}


def _packed_rows(name, n, vocab, dim, group, s, o, scaled=False, pad=0.02, zipf=1.05, tokens="i64"):
    return {"name": name, "kind": "packed_rows", "n": n, "vocab": vocab, "dim": dim, "group": group, "scales": s, "out": o,
            "scaled": scaled, "pad": pad, "zipf": zipf, "tokens": tokens}


def _scores(name, m, vocab, dim, group, s, x, o):
    return {"name": name, "kind": "scores", "m": m, "vocab": vocab, "dim": dim, "group": group, "scales": s, "in": x, "out": o}


def listed():
    return [
        # a decoding step of 8 sequences: latency is all that counts
        _rows("rows_decode", 8, 32000, 1024, "bf16", "bf16", pad=0.0),
        # one prompt of an odd length; fp32 master weights, activations in bf16
        _rows("rows_prompt", 2047, 50001, 768, "f32", "bf16"),
        # a training batch of 32 sequences of 2048 tokens
        _rows("rows_batch", 65536, 131072, 2048, "bf16", "bf16"),
        # a user's history of categories beside the pooled features: a few tokens, narrow rows, the buffer accumulates
        _grad("grad_history", 77, 131072, 64, "f32", "f32", True, tokens="i32"),
        # fine-tuning on two sequences of 2048 tokens: the gradient has the weights' type, and all of it is written
        _grad("grad_tune", 4096, 32000, 1024, "bf16", "bf16", False),
        # ragged batch, a width that no vector divides, gradients of several micro-batches added up in fp32
        _grad("grad_ragged", 30011, 50001, 515, "f16", "f32", True, pad=0.2),
        # pre-training: a quarter of a million tokens, fp32 gradient of the whole vocabulary
        _grad("grad_batch", 262144, 131072, 1024, "bf16", "f32", False),
        # one ranking request: 8 candidates of 26 slots, from a table in 4 bits
        _packed_rows("packed_rows_request", 208, 1 << 20, 64, 32, "f16", "f32"),
        # offline scoring: many tokens, rows of 64 bytes
        _packed_rows("packed_rows_batch", 262144, 1 << 20, 128, 64, "f16", "bf16", tokens="i32"),
        # a request's vector against a small table in fp32: latency
        _scores("scores_small", 1, 4096, 64, 32, "f32", "f32", "f32"),
        # one sequence's next token, an odd vocabulary
        _scores("scores_token", 1, 50001, 1024, 64, "bf16", "bf16", "f32"),
        # eight sequences' next tokens, wide rows
        _scores("scores_eight", 8, 131072, 4096, 128, "f16", "bf16", "bf16"),
    ]


def _spread(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.49)))))))


def _width(rng, low, high):
    """Half of the widths are multiples of 32, the others are any."""
    d = _spread(rng, low, high)
    return d if rng.random() < 0.5 else max(32, d // 32 * 32)


def draw(rng):
    kind = rng.choice(["rows", "grad", "grad", "packed_rows", "scores", "scores"])
    pick = lambda: rng.choice(["f32", "bf16", "f16"])  # noqa: E731
    tokens, pad, zipf = rng.choice(["i32", "i64"]), rng.choice([0.0, 0.03, 0.4]), rng.choice([0.0, 0.9, 1.05, 1.3])
    vocab = _spread(rng, 300, 262144)
    if kind == "rows":
        c = _rows("", _spread(rng, 1, 131072), vocab, _width(rng, 8, 4096), pick(), pick(), rng.random() < 0.7, pad, zipf, tokens)
    elif kind == "grad":
        c = _grad("", _spread(rng, 1, 262144), vocab, _width(rng, 8, 4096), pick(), pick(), rng.random() < 0.5, rng.random() < 0.7,
                  pad, zipf, tokens)
    elif kind == "packed_rows":
        c = _packed_rows("", _spread(rng, 1, 262144), vocab, _width(rng, 8, 4096), rng.choice([32, 64, 128]), pick(), pick(),
                         rng.random() < 0.5, pad, zipf, tokens)
    else:
        c = _scores("", rng.choice([1, 1, 1, 2, 3, 4, 6, 8]), vocab, _width(rng, 8, 8192), rng.choice([32, 64, 128]), pick(),
                    pick(), pick())
    del c["name"]
    if c.get("n", 64) < 64:
        c["pad"] = 0.0           # (a few tokens are not all padding)
    while work(c)["bytes"] > MOST_BYTES or work(c)["flops"] > MOST_FLOPS or c["vocab"] * c["dim"] > 1 << 28:
        k = "n" if c.get("n", 0) * 2 > c["vocab"] else "vocab"
        c[k] = c[k] * 2 // 3
    return c


@functools.lru_cache(maxsize=64)
def _distinct(n, vocab, zipf, pad):
    """How many rows that are not the padding's n tokens are expected to meet."""
    p = np.arange(1, vocab, dtype=np.float64) ** -zipf
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p / p.sum() * (1 - pad), 1 - 1e-12)))))


def work(case):
    c = case
    vocab, dim = c["vocab"], c["dim"]
    if c["kind"] != "scores":
        n = c["n"]
        tokens, met = n * (4 if c["tokens"] == "i32" else 8), _distinct(n, vocab, c["zipf"], c["pad"])
    if c["kind"] in ("packed_rows", "scores"):
        row = (dim + 1) // 2 + -(-dim // c["group"]) * SIZES[c["scales"]]
    if c["kind"] == "rows":
        return {"bytes": tokens + met * dim * SIZES[c["in"]] + n * dim * SIZES[c["out"]], "flops": n * dim}
    if c["kind"] == "grad":
        written = met * 2 if c["add"] else vocab
        return {"bytes": tokens + n * (1 - c["pad"]) * dim * SIZES[c["in"]] + written * dim * SIZES[c["out"]], "flops": n * dim}
    if c["kind"] == "packed_rows":
        return {"bytes": tokens + met * row + n * dim * SIZES[c["out"]], "flops": 2 * n * dim}
    m = c["m"]
    return {"bytes": vocab * row + m * dim * SIZES[c["in"]] + m * vocab * SIZES[c["out"]], "flops": 2.0 * m * vocab * dim}


def _scale(case):
    """The factor as the fp32 number that the call takes."""
    return float(np.float32(math.sqrt(case["dim"]))) if case["scaled"] else 1.0


def _tokens(case, g):
    """Zipf ranks 1 .. vocab - 1 under a permutation of their own, and PADDING."""
    n, vocab = case["n"], case["vocab"]
    p = torch.arange(1, vocab, dtype=torch.float64, device="cuda") ** -case["zipf"]
    edges = torch.cumsum(p, 0)
    u = torch.rand(n, dtype=torch.float64, device="cuda", generator=g) * edges[-1]
    t = 1 + torch.randperm(vocab - 1, device="cuda", generator=g)[torch.searchsorted(edges, u).clamp_(max=vocab - 2)]
    t[torch.rand(n, device="cuda", generator=g) < case["pad"]] = PADDING
    return t.to(torch.int32 if case["tokens"] == "i32" else torch.int64)


def _packed(case, g):
    """Rows in 4 bits: q [vocab, bytes], a row's bytes rounded up to a multiple of 16, and scales [vocab, groups]."""
    vocab, dim, group = case["vocab"], case["dim"], case["group"]
    width = (dim + 31) // 32 * 16
    q = torch.randint(0, 256, (vocab, width), dtype=torch.uint8, device="cuda", generator=g)
    scales = 0.02 * (0.5 + torch.rand((vocab, -(-dim // group)), device="cuda", generator=g))
    return q, scales.to(TYPES[case["scales"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, vocab, dim = case["kind"], case["vocab"], case["dim"]
    s = {"case": case}
    if kind != "scores":
        s["tokens"], s["scale"] = _tokens(case, g), _scale(case)
    if kind == "rows":
        s["weight"] = torch.randn((vocab, dim), device="cuda", generator=g).mul_(0.02).to(TYPES[case["in"]])
        s["out"] = torch.empty((case["n"], dim), dtype=TYPES[case["out"]], device="cuda")
    elif kind == "grad":
        s["grad_out"] = torch.randn((case["n"], dim), device="cuda", generator=g).mul_(0.01).to(TYPES[case["in"]])
        if case["add"]:
            s["grad_weight"] = torch.randn((vocab, dim), device="cuda", generator=g).mul_(0.1).to(TYPES[case["out"]])
        else:
            s["grad_weight"] = torch.empty((vocab, dim), dtype=TYPES[case["out"]], device="cuda")
    else:
        s["q"], s["scales"] = _packed(case, g)
        if kind == "packed_rows":
            s["out"] = torch.empty((case["n"], dim), dtype=TYPES[case["out"]], device="cuda")
        else:
            s["x"] = torch.randn((case["m"], dim), device="cuda", generator=g).to(TYPES[case["in"]])
            s["out"] = torch.empty((case["m"], vocab), dtype=TYPES[case["out"]], device="cuda")
    return s


@functools.lru_cache(maxsize=1)
def _binding():
    from paper_2209_07663_b200 import binding
    return binding


def _own_run(s):
    mb, case = _binding(), s["case"]
    if case["kind"] == "rows":
        mb.mono_token_rows(s["weight"], s["tokens"], s["out"], scale=s["scale"], padding=PADDING)
        return s["out"]
    if case["kind"] == "grad":
        mb.mono_token_rows_grad(s["grad_out"], s["tokens"], s["grad_weight"], scale=s["scale"], padding=PADDING, accumulate=case["add"])
        return s["grad_weight"]
    if case["kind"] == "packed_rows":
        mb.mono_packed_token_rows(s["q"], s["scales"], case["group"], s["tokens"], s["out"], scale=s["scale"], padding=PADDING)
        return s["out"]
    mb.mono_packed_scores(s["q"], s["scales"], case["group"], s["x"], s["out"])
    return s["out"]


def _unpacked(q, scales, group, dim):
    values = torch.stack((q & 15, q >> 4), -1).flatten(1)[:, :dim].float() - 8
    return values * scales.float().repeat_interleave(group, 1)[:, :dim]


def run(state):
    if own:
        return _own_run(state)
    s = state
    case = s["case"]
    out_type = TYPES[case["out"]]
    if case["kind"] == "scores":
        return (s["x"].float() @ _unpacked(s["q"], s["scales"], case["group"], case["dim"]).T).to(out_type)
    tokens = s["tokens"].long()
    there = (tokens >= 0) & (tokens < case["vocab"]) & (tokens != PADDING)
    at = torch.where(there, tokens, 0)
    if case["kind"] == "rows":
        rows = s["weight"][at].float()
    elif case["kind"] == "packed_rows":
        rows = _unpacked(s["q"][at], s["scales"][at], case["group"], case["dim"])
    else:
        terms = torch.where(there[:, None], s["grad_out"].float(), 0.0)
        total = torch.zeros((case["vocab"], case["dim"]), device="cuda").index_add_(0, at, terms).mul_(s["scale"])
        if not case["add"]:
            return total.to(out_type)
        met = torch.zeros(case["vocab"], dtype=torch.bool, device="cuda").index_fill_(0, at, True)
        s["grad_weight"].copy_(torch.where(met[:, None], s["grad_weight"].float() + total, s["grad_weight"].float()))
        return s["grad_weight"]
    return torch.where(there[:, None], rows * s["scale"], 0.0).to(out_type)


def exact(case, seed):
    s = prepare(case, seed)
    dim = case["dim"]
    if case["kind"] in ("packed_rows", "scores"):
        c = torch.arange(dim, device="cuda")

        def values(q, scales):
            return ((q[:, c // 2] >> (4 * (c % 2)).to(torch.uint8)).remainder(16).double() - 8.0) * scales[:, c // case["group"]].double()

        if case["kind"] == "scores":
            step = max(1, (1 << 26) // dim)
            x = s["x"].double()
            parts = [torch.einsum("vc,mc->mv", values(q, scales), x) for q, scales in zip(s["q"].split(step), s["scales"].split(step))]
            return torch.cat(parts, 1)
    keep = (s["tokens"] != PADDING).nonzero()[:, 0]
    tokens = s["tokens"][keep].long()
    if case["kind"] != "grad":
        out = torch.zeros((case["n"], dim), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 26) // dim)
        for at, t in zip(keep.split(step), tokens.split(step)):
            rows = s["weight"][t].double() if case["kind"] == "rows" else values(s["q"][t], s["scales"][t])
            out[at] = rows * s["scale"]
        return out
    # running sums over the tokens in their order, and their differences at the ends of each token's run
    ordered, order = torch.sort(tokens, stable=True)
    out = s["grad_weight"].double() if case["add"] else torch.zeros((case["vocab"], dim), dtype=torch.float64, device="cuda")
    found, counts = torch.unique_consecutive(ordered, return_counts=True)
    if found.numel():
        ends = torch.cumsum(counts, 0)
        for k in range(0, dim, 256):
            sums = torch.cumsum(s["grad_out"][keep[order], k:k + 256].double(), 0)[ends - 1]
            sums[1:] -= sums[:-1].clone()
            out[found, k:k + 256] += sums * s["scale"]
    return out
