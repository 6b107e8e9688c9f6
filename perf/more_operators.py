"""The workloads of the operators between a pruned model's weights and its answers: microscaled
4-bit floating point (packing, and products of tokens with packed weights), and the log
probabilities of given tokens with entropy and top alternatives, with their gradient.

Each case is one call, or the two that belong together, as serving or scoring makes them. With
`own` false, `run` computes it in plain torch operations in 32 bits; with `own` true it calls the
package. Both take the same inputs. Widths are those of `workloads/configs.py` (768, 1000, 4096 and
14336) and odd ones, vocabularies generic; `draw` spreads over the range between them.

Microscaled values: a row is cut into blocks of 32. A block's scale is the power of two 2^(e - 2),
e = floor(log2(max |v|)), not below 2^-127, kept as the byte exponent + 127; a value is v / scale
rounded to the nearest (ties to the even code) of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives,
and at most 6. Code k of a row is in byte k / 2, the even one in the low half; rows are padded with
zero codes to whole 256 values. The scale of block b of the 128 values c is byte
16 (c / 4) + 4 b + c % 4 of its row, and rows of scales are padded to whole 16 bytes.
"""
import math

import torch

own = False

W_STD = 0.015  # of the weights of a block's projections
BLOCK = 32
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
VOCAB = 128000
MOST_FLOPS = 2 * 8192 * 4096 * 14336  # of the largest product
MOST_LOGITS = 8192 * VOCAB
MOST_SORTED = 1024 * VOCAB  # with top alternatives: the plain form sorts whole rows


def listed():
    return [
        # One token of a decoder block on its way to a packed product. Latency.
        {"name": "mx4 pack token", "kind": "pack", "n": 1, "d": 4096, "dtype": "bf16", "pad": 0},
        # An up projection after its solve, rounded to its packed values.
        {"name": "mx4 pack weights", "kind": "pack", "n": 14336, "d": 4096, "dtype": "f32",
         "pad": 0},
        # One token, 16-bit, through a down projection: the weights are read.
        {"name": "mx4 token", "kind": "linear", "n": 1, "d": 14336, "ff": 4096, "x": "bf16",
         "out": "bf16"},
        # A few tokens of a small layer with odd widths.
        {"name": "mx4 few ragged", "kind": "linear", "n": 13, "d": 1001, "ff": 2731, "x": "bf16",
         "out": "f32"},
        # The output head for a batch of 64 sequences, its tokens packed too.
        {"name": "mx4 head", "kind": "linear", "n": 64, "d": 4096, "ff": VOCAB, "x": "mx4",
         "out": "bf16"},
        # A short prompt through odd widths.
        {"name": "mx4 prompt ragged", "kind": "linear", "n": 777, "d": 4097, "ff": 5001,
         "x": "mx4", "out": "bf16"},
        # Four sequences of 2048 tokens through an up projection.
        {"name": "mx4 prompts", "kind": "linear", "n": 8192, "d": 4096, "ff": 14336, "x": "mx4",
         "out": "bf16"},
        # One decoded token: its log probability and 20 alternatives. Latency.
        {"name": "logprobs token", "kind": "logprobs", "n": 1, "vocab": VOCAB, "dtype": "bf16",
         "top": 20, "masked": False, "pad": 0, "scale": 1.0},
        # Scoring four sequences of 2048 tokens, as for perplexity.
        {"name": "logprobs scoring", "kind": "logprobs", "n": 8192, "vocab": VOCAB,
         "dtype": "bf16", "top": 0, "masked": False, "pad": 0, "scale": 1.0},
        # Answers under a grammar's mask at a temperature, fp32 logits out of wider rows.
        {"name": "logprobs ragged", "kind": "logprobs", "n": 301, "vocab": 50001, "dtype": "f32",
         "top": 8, "masked": True, "pad": 3, "scale": 1.25},
        # The loss's gradient over two sequences, with a term in the entropy.
        {"name": "logprobs backward", "kind": "logprobs_grad", "n": 4096, "vocab": VOCAB,
         "dtype": "bf16", "masked": False, "pad": 0, "scale": 1.0},
        # The same of fp32 logits, odd sizes, under a mask.
        {"name": "logprobs backward ragged", "kind": "logprobs_grad", "n": 301, "vocab": 50001,
         "dtype": "f32", "masked": True, "pad": 3, "scale": 1.25},
    ]


def _spread(rng, lo, hi):
    """A size from lo to hi, even in its logarithm; every second one a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v -= v % 64
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["pack", "linear", "linear", "linear", "logprobs", "logprobs",
                       "logprobs_grad"])
    if kind == "pack":
        d = _spread(rng, 32, 14336)
        return {"kind": kind, "n": _spread(rng, 1, 14336 * 4096 // d), "d": d,
                "dtype": rng.choice(["bf16", "f32"]), "pad": rng.choice([0, 0, 3, 8])}
    if kind == "linear":
        d, ff = _spread(rng, 64, 14336), _spread(rng, 64, 14336)
        x = rng.choice(["bf16", "mx4", "mx4"])
        few = x == "bf16" or rng.random() < 0.4
        n = _spread(rng, 1, 64) if few else _spread(rng, 64, min(32768, MOST_FLOPS // (2 * d * ff)))
        return {"kind": kind, "n": n, "d": d, "ff": ff, "x": x,
                "out": rng.choice(["bf16", "bf16", "f32"])}
    vocab, top = _spread(rng, 64, VOCAB), 0
    if kind == "logprobs":
        top = rng.choice([0, 0, 1, 5, 20, 32])
    most = MOST_SORTED if top else MOST_LOGITS // (2 if kind == "logprobs_grad" else 1)
    dtype = rng.choice(["bf16", "f32"])
    case = {"kind": kind, "n": _spread(rng, 1, min(65536, most // (2 if dtype == "f32" else 1) //
                                                   vocab)),
            "vocab": vocab, "dtype": dtype}
    if kind == "logprobs":
        case["top"] = top
    case["masked"] = vocab >= 1024 and rng.random() < 0.5
    case["pad"] = rng.choice([0, 0, 3, 8])
    case["scale"] = rng.choice([1.0, 1.0, 1.25, 0.5])
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _activations(g, n, d):
    """Tokens with heavy tails and eight channels that are larger than the rest."""
    x = torch.randn(n, d, generator=g, device="cuda")
    x *= torch.exp(0.5 * torch.randn(n, 1, generator=g, device="cuda"))
    x[:, torch.randint(0, d, (8,), generator=g, device="cuda")] *= 10.0
    return x


def _weights(g, n, d):
    """Half of the entries are zero, as after the solve."""
    w = W_STD * torch.randn(n, d, generator=g, device="cuda")
    w *= torch.rand(n, d, generator=g, device="cuda") < 0.5
    return w


def _microscaled(v):
    """Values, magnitudes' codes and scale exponents of rows v by the rule at the top of this
    file: [n, blocks, 32] twice and [n, blocks]."""
    n, d = v.shape
    wide = torch.nn.functional.pad(v.float(), (0, -d % BLOCK)).view(n, -1, BLOCK)
    top = wide.abs().amax(2)
    _, e = torch.frexp(top)  # top = m 2^e, m in [0.5, 1)
    e = torch.where(top > 0, torch.clamp(e - 1 - 2, min=-127), -127)
    # In two factors: 2^127 is the largest power of two in 32 bits, and 2^-127 no normal number.
    half = torch.div(e, 2, rounding_mode="floor")
    u = wide * torch.exp2(-half.float()).unsqueeze(2) * torch.exp2((half - e).float()).unsqueeze(2)
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.clamp(torch.round(a / step) * step, max=6.0)
    values = torch.copysign(a, u) * torch.exp2(half.float()).unsqueeze(2) * \
        torch.exp2((e - half).float()).unsqueeze(2)
    return values, torch.copysign(a, u), e


def _pack(v):
    """Codes and scales of rows v, in the layout at the top of this file."""
    n, d = v.shape
    _, units, e = _microscaled(v)
    levels = torch.tensor(LEVELS, device=v.device)
    codes = torch.searchsorted(levels, units.abs().contiguous()).to(torch.uint8)
    codes = codes + 8 * (units < 0).to(torch.uint8)
    codes = codes.view(n, -1)
    codes = torch.nn.functional.pad(codes, (0, -codes.shape[1] % 256)).view(n, -1, 2)
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 16))
    s = s.view(n, -1, 4, 4).transpose(2, 3).reshape(n, -1)  # 128 values, block -> block, 128 values
    return (codes[..., 0] | (codes[..., 1] << 4)).contiguous(), s.contiguous()


def _packed_like(n, d):
    """Room for the codes and scales of n rows of d."""
    return (torch.empty(n, -(-d // 256) * 128, dtype=torch.uint8, device="cuda"),
            torch.empty(n, -(-d // 512) * 16, dtype=torch.uint8, device="cuda"))


def _logits(g, n, case):
    """Logits of a trained head: a spread of 2.5, and in each row a few that stand out."""
    v, dt = case["vocab"], DTYPES[case["dtype"]]
    x = torch.randn(n, v + case["pad"], generator=g, device="cuda", dtype=torch.float32)
    x *= 2.5
    at = torch.randint(0, v, (n, 1), generator=g, device="cuda")
    at = (at + v // 4 * torch.arange(4, device="cuda")) % v
    x.scatter_add_(1, at, 4 + 4 * torch.rand(n, 4, generator=g, device="cuda"))
    tokens = torch.randint(0, v, (n,), generator=g, device="cuda")
    likely = torch.rand(n, generator=g, device="cuda") < 0.5
    tokens = torch.where(likely, at[:, 0], tokens)
    if case["masked"]:
        x[:, :v].masked_fill_(torch.rand(v, generator=g, device="cuda") < 0.4, float("-inf"))
        x.scatter_(1, tokens.unsqueeze(1), 3.0)
    # Some rows have no token to score: padding of a batch.
    tokens[torch.rand(n, generator=g, device="cuda") < 0.05] = -100
    return x.to(dt)[:, :v], tokens


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, n = case["kind"], case["n"]
    st = dict(case)
    if kind == "pack":
        st["X"] = _activations(g, n, case["d"] + case["pad"]).to(DTYPES[case["dtype"]])[:, :case["d"]]
        st["Q"], st["scales"] = _packed_like(n, case["d"])
        st["Y"] = torch.empty(n, case["d"], dtype=torch.bfloat16, device="cuda")
    elif kind == "linear":
        st["X"] = _activations(g, n, case["d"]).to(torch.bfloat16)
        st["Q"], st["scales"] = _pack(_weights(g, case["ff"], case["d"]))
        if case["x"] == "mx4":
            st["XQ"], st["x_scales"] = _packed_like(n, case["d"])
        st["Y"] = torch.empty(n, case["ff"], dtype=DTYPES[case["out"]], device="cuda")
    else:
        st["logits"], st["tokens"] = _logits(g, n, case)
        if kind == "logprobs":
            for name in ("logp", "lse", "entropy"):
                st[name] = torch.empty(n, device="cuda")
            st["top_index"] = st["top_logp"] = None
            if case["top"]:
                st["top_index"] = torch.empty(n, case["top"], dtype=torch.int64, device="cuda")
                st["top_logp"] = torch.empty(n, case["top"], device="cuda")
        else:
            _, st["lse"], st["entropy"] = _distribution(st)
            # A policy's gradient: of either sign, with an entropy bonus and a pull on lse.
            st["dlogp"] = torch.randn(n, generator=g, device="cuda")
            st["dentropy"] = 0.1 * torch.randn(n, generator=g, device="cuda")
            st["dlse"] = 0.01 * torch.randn(n, generator=g, device="cuda")
            st["dlogits"] = torch.empty(n, case["vocab"], dtype=DTYPES[case["dtype"]],
                                        device="cuda")
    st["ws"] = None  # a workspace, once a call has asked for one
    return st


# ---------------------------------------------------------------------------
# One pass: the package's calls
# ---------------------------------------------------------------------------


def _ws(st, nbytes):
    if st["ws"] is None:
        st["ws"] = torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")
    return st["ws"]


def _run_own(st):
    import paper_2512_13886_amd as L
    kind = st["kind"]
    if kind == "pack":
        L.optima_mx4_pack(st["X"], st["Q"], st["scales"])
        L.optima_mx4_unpack(st["Q"], st["scales"], st["Y"])
        return {"Y": st["Y"]}
    if kind == "linear":
        X, x_scales = st["X"], None
        if st["x"] == "mx4":
            L.optima_mx4_pack(X, st["XQ"], st["x_scales"])
            X, x_scales = st["XQ"], st["x_scales"]
        ws = _ws(st, L.optima_mx4_workspace_bytes(st["n"], st["d"], st["ff"]))
        L.optima_mx4_linear(X, st["Q"], st["scales"], st["Y"], x_scales=x_scales, ws=ws)
        return {"Y": st["Y"]}
    if kind == "logprobs":
        ws = _ws(st, L.optima_token_logprobs_workspace_bytes(st["n"], st["vocab"], st["top"]))
        L.optima_token_logprobs(st["logits"], st["tokens"], st["logp"], lse=st["lse"],
                                entropy=st["entropy"], top_index=st["top_index"],
                                top_logp=st["top_logp"], scale=st["scale"], ws=ws)
        return {k: st[k] for k in ("logp", "lse", "entropy", "top_index", "top_logp")}
    L.optima_token_logprobs_backward(st["logits"], st["lse"], st["dlogits"], tokens=st["tokens"],
                                     dlogp=st["dlogp"], entropy=st["entropy"],
                                     dentropy=st["dentropy"], dlse=st["dlse"], scale=st["scale"])
    return {"dlogits": st["dlogits"]}


# ---------------------------------------------------------------------------
# One pass: the plain form
# ---------------------------------------------------------------------------


def _unpack(Q, scales, d):
    """The weights that codes and scales stand for, float32 [n, d]."""
    n = Q.shape[0]
    codes = torch.stack([Q & 15, Q >> 4], 2).view(n, -1)[:, :d].long()
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=Q.device)
    e = scales.view(n, -1, 4, 4).transpose(2, 3).reshape(n, -1).float() - 127.0
    return levels[codes] * torch.repeat_interleave(torch.exp2(e), BLOCK, 1)[:, :d]


def _distribution(st):
    """Scaled logits, lse and entropy, float32."""
    z = st["logits"].float() * st["scale"]
    top = z.amax(1, keepdim=True)
    y = z - top
    e = torch.exp(y)
    total = e.sum(1)
    mean = torch.where(e > 0, e * y, 0.0).sum(1) / total
    return z, top.squeeze(1) + torch.log(total), torch.log(total) - mean


def _run_plain(st):
    kind = st["kind"]
    if kind == "pack":
        values, _, _ = _microscaled(st["X"])
        return {"Y": values.view(st["n"], -1)[:, :st["d"]].to(torch.bfloat16)}
    if kind == "linear":
        x = st["X"].float()
        if st["x"] == "mx4":
            x = _microscaled(x)[0].view(st["n"], -1)[:, :st["d"]]
        y = x @ _unpack(st["Q"], st["scales"], st["d"]).t()
        return {"Y": y.to(DTYPES[st["out"]])}
    tokens, given = st["tokens"], st["tokens"] >= 0
    if kind == "logprobs":
        z, lse, entropy = _distribution(st)
        zt = torch.gather(z, 1, tokens.clamp(min=0).unsqueeze(1)).squeeze(1)
        out = {"logp": torch.where(given, zt - lse, 0.0), "lse": lse, "entropy": entropy,
               "top_index": None, "top_logp": None}
        if st["top"]:  # equal ones in the order of their indices
            best, at = torch.sort(z, dim=1, descending=True, stable=True)
            out["top_index"] = at[:, :st["top"]].contiguous()
            out["top_logp"] = best[:, :st["top"]] - lse.unsqueeze(1)
        return out
    z = st["logits"].float() * st["scale"]
    logp = z - st["lse"].unsqueeze(1)
    p = torch.exp(logp)
    g = torch.where(given, st["dlogp"], 0.0).unsqueeze(1)
    slope = torch.where(p > 0, logp + st["entropy"].unsqueeze(1), 0.0)
    dz = p * (st["dlse"].unsqueeze(1) - g - st["dentropy"].unsqueeze(1) * slope)
    dz.scatter_add_(1, tokens.clamp(min=0).unsqueeze(1), g)
    return {"dlogits": (dz * st["scale"]).to(st["logits"].dtype)}


def run(st):
    return _run_own(st) if own else _run_plain(st)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    kind, n = case["kind"], case["n"]
    if kind == "pack":
        d, e = case["d"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * d * (e + 2) + n * (d / 2 + -(-d // BLOCK)), "flops": 4 * n * d}
    if kind == "linear":
        d, ff = case["d"], case["ff"]
        return {"bytes": ff * (d / 2 + -(-d // BLOCK)) + 2 * n * d +
                (2 if case["out"] == "bf16" else 4) * n * ff, "flops": 2 * n * d * ff}
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "logprobs":
        return {"bytes": n * (e * case["vocab"] + 8 + 12 + 12 * case["top"]),
                "flops": 6 * n * case["vocab"]}
    return {"bytes": n * (2 * e * case["vocab"] + 8 + 20), "flops": 8 * n * case["vocab"]}


def _exact_values(v):
    """Rows v as microscaled values in 64 bits, by the intervals of values that each code takes."""
    n, d = v.shape
    of = torch.arange(d, device=v.device) // BLOCK
    top = torch.zeros(n, int(of[-1]) + 1, dtype=torch.float64, device=v.device)
    top.scatter_reduce_(1, of.expand(n, d), v.double().abs(), "amax")
    e = torch.log2(top.clamp(min=2.0 ** -160)).floor()
    # Where the logarithm rounds up to a whole number.
    e = torch.where(torch.pow(2.0, e) > top, e - 1, e)
    scale = torch.pow(2.0, (e - 2).clamp(min=-127.0))[:, of]
    u = v.double() / scale
    a, out = u.abs(), torch.zeros_like(u)
    # Borders between neighbours; a value on one goes to the neighbour with the even code.
    for k in range(1, 8):
        border = (LEVELS[k - 1] + LEVELS[k]) / 2
        out = torch.where(a >= border if k % 2 == 0 else a > border, LEVELS[k], out)
    return torch.where(u < 0, -out, out) * scale


def _exact_weights(Q, scales, d):
    """Value of every weight, by index: where in its row value k is kept."""
    k = torch.arange(d, device=Q.device)
    byte = Q[:, k // 2].long()
    code = torch.where(k % 2 == 1, byte // 16, byte % 16)
    low = code % 8
    size = torch.where(low < 2, low * 0.5, (1 + (low % 2) * 0.5) * torch.pow(2.0, low // 2 - 1))
    c, b = k // 128, k % 128 // 32
    e = scales[:, 16 * (c // 4) + 4 * b + c % 4].double() - 127
    return torch.where(code >= 8, -size, size).double() * torch.pow(2.0, e)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "pack":
        return {"Y": _exact_values(st["X"])}
    if kind == "linear":
        x = _exact_values(st["X"]) if case["x"] == "mx4" else st["X"].double()
        w = _exact_weights(st["Q"], st["scales"], case["d"])
        return {"Y": torch.mm(x, w.t().contiguous())}
    z = st["logits"].double() * case["scale"]
    tokens = st["tokens"]
    rows = torch.nonzero(tokens >= 0).squeeze(1)
    if kind == "logprobs":
        lse = torch.logsumexp(z, 1)
        p = torch.softmax(z, 1)
        out = {"logp": torch.zeros_like(lse), "lse": lse,
               "entropy": torch.special.entr(p).sum(1), "top_index": None, "top_logp": None}
        out["logp"][rows] = z[rows, tokens[rows]] - lse[rows]
        if case["top"]:
            out["top_logp"] = torch.topk(z, case["top"], 1).values - lse.unsqueeze(1)
        return out
    # From the definition: d lse = p, d H = -p (log p + H), d logp = onehot - p, at the lse and
    # entropy that the call is given.
    logp = z - st["lse"].double().unsqueeze(1)
    p = torch.exp(logp)
    g = torch.zeros_like(st["dlse"], dtype=torch.float64)
    g[rows] = st["dlogp"][rows].double()
    dz = (st["dlse"].double() - g).unsqueeze(1) * p
    dz -= st["dentropy"].double().unsqueeze(1) * (st["entropy"].double().unsqueeze(1) * p -
                                                  torch.special.entr(p))
    dz[rows, tokens[rows]] += g[rows]
    return {"dlogits": dz * case["scale"]}
