"""The workloads of the feed-forward operators: the RMS norm with the residual's
addition (its output in 16, 32 or 8 bits, and its gradient), the gated product
of the gate and up projections (and its gradient), and products with 4-bit
weights.

Each case is one call as pruning, recovering or serving the feed-forward half of
a decoder block makes it. With `own` false, `run` computes it in plain torch
operations in 32 bits; with `own` true it calls the package. Both take the same
inputs. Sizes are those of `workloads/configs.py` (768, 1000, 4096 and 14336 wide)
and odd ones; `draw` spreads over the range between them.

4-bit weights: row n of W [n, d] is cut into groups of `group` values with one
bfloat16 scale each, scale = bf16(max |w| / 7), code = clamp(rne(w / scale), -7, 7).
A chunk of 128 codes takes 64 bytes: dword j of the 16-byte block b holds the codes
32 j + 8 b .. + 7, the even ones in nibbles 0..3 and the odd ones in nibbles 4..7,
each as code + 8. Rows are padded to whole chunks with zero codes.
"""
import math

import torch

own = False

EPS = 1e-6
W_STD = 0.015  # of the weights of the block's projections
CHUNK = 128
NIBBLE_OF = [0, 4, 1, 5, 2, 6, 3, 7]  # the nibble that holds code k of eight
MOST_FLOPS = 4 * 8192 * 4096 * 14336  # of the largest listed case
MOST_VALUES = 32768 * 4096


def listed():
    return [
        # One token of a decoder block on its way to 8-bit products: the
        # residual's addition, the norm and one scale for 128 values. Latency.
        {"name": "norm token 8-bit", "kind": "norm", "n": 1, "d": 4096, "dtype": "bf16",
         "residual": True, "out": "i8", "group": 128, "pad": 0},
        # The inputs of the gate and up projections over 16 calibration
        # sequences of 2048 tokens, from which their Hessian is formed.
        {"name": "norm calibration", "kind": "norm", "n": 32768, "d": 4096, "dtype": "bf16",
         "residual": True, "out": "bf16", "group": 0, "pad": 0},
        # A layer kept in fp32 whose sizes are no multiple of anything, read out
        # of wider rows; one 8-bit scale a token.
        {"name": "norm fp32 ragged", "kind": "norm", "n": 20001, "d": 1001, "dtype": "f32",
         "residual": False, "out": "i8", "group": 0, "pad": 3},
        # The gradient of the norm in a recovery step over 8 sequences.
        {"name": "norm backward", "kind": "norm_grad", "n": 16384, "d": 4096, "dtype": "bf16",
         "residual": True},
        # One token through the gate and up projections: both weights are read.
        {"name": "gated token", "kind": "gated", "n": 1, "d": 4096, "ff": 14336, "saved": False},
        # A few tokens of a small layer with odd widths.
        {"name": "gated few ragged", "kind": "gated", "n": 13, "d": 1001, "ff": 2731,
         "saved": False},
        # The forward pass of a recovery step over 4 sequences, which keeps
        # both projections for the gradient.
        {"name": "gated forward", "kind": "gated", "n": 8192, "d": 4096, "ff": 14336,
         "saved": True},
        # Its gradient over 2 sequences.
        {"name": "gated backward", "kind": "gated_grad", "n": 4096, "d": 4096, "ff": 14336,
         "masked": False},
        # The same for odd sizes, the weights' gradients under their masks.
        {"name": "gated backward ragged", "kind": "gated_grad", "n": 1999, "d": 1001, "ff": 2731,
         "masked": True},
        # One token with 4-bit weights and the 8-bit output of the norm.
        {"name": "4-bit gated token", "kind": "w4_gated", "n": 1, "d": 4096, "ff": 14336,
         "group": 128, "x": "i8", "x_group": 128},
        # The down projection of eight tokens, 16-bit activations, finer groups.
        {"name": "4-bit down", "kind": "w4", "n": 8, "d": 14336, "ff": 4096, "group": 64,
         "x": "bf16", "x_group": 0},
        # Laying out the weights of an up projection after its solve.
        {"name": "4-bit pack", "kind": "w4_pack", "d": 4096, "ff": 14336, "group": 128,
         "dtype": "f32"},
    ]


def _spread(rng, lo, hi):
    """A size from lo to hi, even in its logarithm; every second one a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and v >= 64:
        v -= v % 64
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_grad", "gated", "gated", "gated_grad", "w4",
                       "w4_gated", "w4_pack"])
    if kind in ("norm", "norm_grad"):
        d = _spread(rng, 64, 14336)
        most = MOST_VALUES if kind == "norm" else 16384 * 4096
        case = {"kind": kind, "n": _spread(rng, 1, most // d), "d": d,
                "dtype": rng.choice(["bf16", "bf16", "f32"]), "residual": rng.random() < 0.6}
        if kind == "norm":
            case["out"] = rng.choice(["bf16", "f32", "i8"])
            case["group"] = rng.choice([0, 32, 64, 128]) if case["out"] == "i8" else 0
            case["pad"] = rng.choice([0, 0, 3, 8])
        return case
    if kind in ("gated", "gated_grad"):
        d, ff = _spread(rng, 64, 4096), _spread(rng, 64, 14336)
        few = kind == "gated" and rng.random() < 0.5
        most = min(32768, MOST_FLOPS // ((4 if kind == "gated" else 8) * d * ff))
        n = _spread(rng, 1, 64) if few else _spread(rng, 64, max(64, most))
        case = {"kind": kind, "n": n, "d": d, "ff": ff}
        case["saved" if kind == "gated" else "masked"] = rng.random() < 0.5
        return case
    d, ff = _spread(rng, 64, 14336), _spread(rng, 64, 14336)
    case = {"kind": kind, "d": d, "ff": ff, "group": rng.choice([32, 64, 128])}
    if kind == "w4_pack":
        case["dtype"] = rng.choice(["f32", "bf16"])
        return case
    case["n"] = _spread(rng, 1, 64)
    case["x"] = rng.choice(["bf16", "i8"])
    case["x_group"] = rng.choice([0, case["group"]]) if case["x"] == "i8" else 0
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}


def _activations(g, n, d, scale=1.0):
    """Tokens with heavy tails and eight channels that are larger than the rest."""
    x = torch.randn(n, d, generator=g, device="cuda")
    x *= scale * torch.exp(0.5 * torch.randn(n, 1, generator=g, device="cuda"))
    x[:, torch.randint(0, d, (8,), generator=g, device="cuda")] *= 10.0
    return x


def _weights(g, n, d, pruned=False):
    w = W_STD * torch.randn(n, d, generator=g, device="cuda")
    if pruned:  # half of the entries are zero, as after the solve
        w *= torch.rand(n, d, generator=g, device="cuda") < 0.5
    return w


def _pack(w, group):
    """Codes and scales of w by the rule at the top of this file, in its layout."""
    n, d = w.shape
    width = -(-d // group) * group
    wide = torch.nn.functional.pad(w.float(), (0, width - d)).view(n, -1, group)
    scales = (wide.abs().amax(2) / 7.0).bfloat16()
    s = scales.float().unsqueeze(2)
    codes = torch.where(s > 0, torch.clamp(torch.round(wide / s), -7, 7), torch.zeros_like(wide))
    codes = codes.view(n, width)[:, :d].to(torch.int16) + 8
    rows = -(-d // CHUNK) * CHUNK
    codes = torch.nn.functional.pad(codes, (0, rows - d), value=8).to(torch.uint8)
    codes = codes.view(n, -1, 4, 4, 8).transpose(2, 3)  # chunk, block, dword, code
    codes = codes[..., [NIBBLE_OF.index(i) for i in range(8)]].reshape(n, -1, 2)
    return (codes[..., 0] | (codes[..., 1] << 4)).contiguous(), scales.contiguous()


def _eight_bits(x, group):
    """Codes and scales of activations, one scale for `group` values (0: a token)."""
    n, d = x.shape
    group = group or d
    width = -(-d // group) * group
    wide = torch.nn.functional.pad(x, (0, width - d)).view(n, -1, group)
    scales = wide.abs().amax(2) / 127.0
    s = scales.unsqueeze(2)
    codes = torch.where(s > 0, torch.round(wide / s), torch.zeros_like(wide))
    return codes.view(n, width)[:, :d].to(torch.int8).contiguous(), scales.contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, d = case["kind"], case["d"]
    st = dict(case)
    if kind in ("norm", "norm_grad"):
        n, dt = case["n"], DTYPES[case["dtype"]]
        st["weight"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
        if kind == "norm":
            wide = d + case["pad"]
            st["X"] = _activations(g, n, wide).to(dt)[:, :d]
            st["R"] = _activations(g, n, wide).to(dt)[:, :d] if case["residual"] else None
            st["S"] = torch.empty(n, d, dtype=dt, device="cuda") if case["residual"] else None
            st["Y"] = torch.empty(n, d, dtype=DTYPES[case["out"]], device="cuda")
            st["scales"] = None
            if case["out"] == "i8":
                groups = -(-d // case["group"]) if case["group"] else 1
                st["scales"] = torch.empty(n, groups, device="cuda")
        else:
            st["S"] = _activations(g, n, d).to(dt)
            st["dY"] = _activations(g, n, d, 0.01).to(dt)
            st["dS"] = _activations(g, n, d, 0.01).to(dt) if case["residual"] else None
            st["dX"] = torch.empty(n, d, dtype=dt, device="cuda")
            st["dweight"] = torch.empty(d, device="cuda")
    elif kind in ("gated", "gated_grad"):
        n, ff, b = case["n"], case["ff"], torch.bfloat16
        st["X"] = _activations(g, n, d).to(b)
        st["Wg"], st["Wu"] = _weights(g, ff, d).to(b), _weights(g, ff, d).to(b)
        if kind == "gated":
            st["H"] = torch.empty(n, ff, dtype=b, device="cuda")
            st["G"] = torch.empty(n, ff, dtype=b, device="cuda") if case["saved"] else None
            st["U"] = torch.empty(n, ff, dtype=b, device="cuda") if case["saved"] else None
        else:
            st["G"] = (st["X"].float() @ st["Wg"].float().t()).to(b)
            st["U"] = (st["X"].float() @ st["Wu"].float().t()).to(b)
            st["dH"] = _activations(g, n, ff, 0.01).to(b)
            st["dX"] = torch.empty(n, d, dtype=b, device="cuda")
            st["dWg"] = torch.empty(ff, d, dtype=b, device="cuda")
            st["dWu"] = torch.empty(ff, d, dtype=b, device="cuda")
            st["mask_g"] = st["mask_u"] = None
            if case["masked"]:
                st["mask_g"] = (torch.rand(ff, d, generator=g, device="cuda") < 0.5).to(torch.uint8)
                st["mask_u"] = (torch.rand(ff, d, generator=g, device="cuda") < 0.5).to(torch.uint8)
    elif kind == "w4_pack":
        st["W"] = _weights(g, case["ff"], d, True).to(DTYPES[case["dtype"]])
        st["Q"] = torch.empty(case["ff"], -(-d // CHUNK) * CHUNK // 2, dtype=torch.uint8,
                              device="cuda")
        st["scales"] = torch.empty(case["ff"], -(-d // case["group"]), dtype=torch.bfloat16,
                                   device="cuda")
    else:
        x = _activations(g, case["n"], d)
        st["X"], st["x_scales"] = x.to(torch.bfloat16), None
        if case["x"] == "i8":
            st["X"], st["x_scales"] = _eight_bits(x, case["x_group"])
        st["Q"], st["scales"] = _pack(_weights(g, case["ff"], d, True), case["group"])
        if kind == "w4_gated":
            st["Q2"], st["scales2"] = _pack(_weights(g, case["ff"], d, True), case["group"])
        st["Y"] = torch.empty(case["n"], case["ff"], dtype=torch.bfloat16, device="cuda")
    st["ws"] = None  # a workspace, once a call has asked for one
    return st


# ---------------------------------------------------------------------------
# One pass: the package's calls
# ---------------------------------------------------------------------------


def _values(Y, scales, group):
    """What 8-bit codes stand for, in the 16-bit type of activations."""
    if scales is None:
        return Y
    d = Y.shape[1]
    each = torch.repeat_interleave(scales, group, 1)[:, :d] if group else scales
    return (Y.float() * each).bfloat16()


def _ws(L, st, nbytes):
    if st["ws"] is None:
        st["ws"] = torch.empty(max(nbytes, 1), dtype=torch.uint8, device="cuda")
    return st["ws"]


def _run_own(st):
    import paper_2512_13886_amd as L
    kind = st["kind"]
    if kind == "norm":
        L.optima_rms_norm(st["X"], st["weight"], st["Y"], eps=EPS, R=st["R"], S=st["S"],
                          scales=st["scales"], group=st["group"])
        return {"S": st["S"], "Y": _values(st["Y"], st["scales"], st["group"]),
                "scales": st["scales"]}
    if kind == "norm_grad":
        ws = _ws(L, st, L.optima_rms_norm_backward_workspace_bytes(st["n"], st["d"]))
        L.optima_rms_norm_backward(st["S"], st["weight"], st["dY"], st["dX"], eps=EPS,
                                   dS=st["dS"], dweight=st["dweight"], ws=ws)
        return {"dX": st["dX"], "dweight": st["dweight"]}
    if kind == "gated":
        ws = _ws(L, st, L.optima_gated_forward_workspace_bytes(st["n"], st["d"], st["ff"]))
        L.optima_gated_forward(st["X"], st["Wg"], st["Wu"], st["H"], act=L.ACT_SILU, G=st["G"],
                               U=st["U"], ws=ws)
        return {"H": st["H"], "G": st["G"], "U": st["U"]}
    if kind == "gated_grad":
        ws = _ws(L, st, L.optima_gated_backward_workspace_bytes(st["n"], st["d"], st["ff"]))
        L.optima_gated_backward(st["X"], st["Wg"], st["Wu"], st["G"], st["U"], st["dH"],
                                dX=st["dX"], dWg=st["dWg"], dWu=st["dWu"], act=L.ACT_SILU,
                                mask_g=st["mask_g"], mask_u=st["mask_u"], ws=ws)
        return {"dX": st["dX"], "dWg": st["dWg"], "dWu": st["dWu"]}
    if kind == "w4":
        L.optima_w4_linear(st["X"], st["Q"], st["scales"], st["Y"], group=st["group"],
                           x_scales=st["x_scales"], x_group=st["x_group"])
        return {"Y": st["Y"]}
    if kind == "w4_gated":
        L.optima_w4_gated(st["X"], st["Q"], st["scales"], st["Q2"], st["scales2"], st["Y"],
                          group=st["group"], act=L.ACT_SILU, x_scales=st["x_scales"],
                          x_group=st["x_group"])
        return {"Y": st["Y"]}
    L.optima_w4_pack(st["W"], st["Q"], st["scales"], group=st["group"])
    return {"Q": st["Q"], "scales": st["scales"]}


# ---------------------------------------------------------------------------
# One pass: the plain form
# ---------------------------------------------------------------------------


def _unpack(Q, scales, group, d):
    """The weights that 4-bit codes stand for, float32 [n, d]."""
    n = Q.shape[0]
    codes = torch.stack([Q & 15, Q >> 4], 2).view(n, -1, 4, 4, 8)[..., NIBBLE_OF]
    codes = codes.transpose(2, 3).reshape(n, -1)[:, :d].float() - 8.0
    return codes * torch.repeat_interleave(scales.float(), group, 1)[:, :d]


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _run_plain(st):
    kind = st["kind"]
    if kind == "norm":
        s = st["X"].float()
        if st["R"] is not None:
            s = s + st["R"].float()
        y = s * torch.rsqrt((s * s).mean(1, keepdim=True) + EPS) * st["weight"].float()
        S = s.to(st["X"].dtype) if st["R"] is not None else None
        if st["out"] != "i8":
            return {"S": S, "Y": y.to(DTYPES[st["out"]]), "scales": None}
        codes, scales = _eight_bits(y, st["group"])
        return {"S": S, "Y": _values(codes, scales, st["group"]), "scales": scales}
    if kind == "norm_grad":
        s, dy, w = st["S"].float(), st["dY"].float(), st["weight"].float()
        rstd = torch.rsqrt((s * s).mean(1, keepdim=True) + EPS)
        xh, p = s * rstd, dy * w
        dx = rstd * (p - xh * (p * xh).mean(1, keepdim=True))
        if st["dS"] is not None:
            dx = dx + st["dS"].float()
        return {"dX": dx.to(st["S"].dtype), "dweight": (dy * xh).sum(0)}
    if kind == "gated":
        x = st["X"].float()
        g, u = x @ st["Wg"].float().t(), x @ st["Wu"].float().t()
        h = (_silu(g) * u).bfloat16()
        return {"H": h, "G": g.bfloat16() if st["saved"] else None,
                "U": u.bfloat16() if st["saved"] else None}
    if kind == "gated_grad":
        x, wg, wu = st["X"].float(), st["Wg"].float(), st["Wu"].float()
        g, u, dh = st["G"].float(), st["U"].float(), st["dH"].float()
        sig = 1.0 / (1.0 + torch.exp(-g))
        du = dh * g * sig
        dg = dh * u * sig * (1.0 + g * (1.0 - sig))
        dx = dg @ wg + du @ wu
        dwg, dwu = dg.t() @ x, du.t() @ x
        if st["mask_g"] is not None:
            dwg, dwu = dwg * st["mask_g"], dwu * st["mask_u"]
        return {"dX": dx.bfloat16(), "dWg": dwg.bfloat16(), "dWu": dwu.bfloat16()}
    if kind == "w4_pack":
        Q, scales = _pack(st["W"], st["group"])
        return {"Q": Q, "scales": scales}
    x = st["X"].float()
    if st["x_scales"] is not None:
        group = st["x_group"]
        x = x * (torch.repeat_interleave(st["x_scales"], group, 1)[:, :st["d"]] if group
                 else st["x_scales"])
    y = x @ _unpack(st["Q"], st["scales"], st["group"], st["d"]).t()
    if kind == "w4_gated":
        y = _silu(y) * (x @ _unpack(st["Q2"], st["scales2"], st["group"], st["d"]).t())
    return {"Y": y.bfloat16()}


def run(st):
    return _run_own(st) if own else _run_plain(st)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and its result in 64 bits
# ---------------------------------------------------------------------------


def work(case):
    kind, d = case["kind"], case["d"]
    if kind in ("norm", "norm_grad"):
        n, e = case["n"], 2 if case["dtype"] == "bf16" else 4
        if kind == "norm_grad":
            return {"bytes": n * d * e * (4 if case["residual"] else 3) + d * (e + 4),
                    "flops": 11 * n * d}
        out = {"bf16": 2, "f32": 4, "i8": 1}[case["out"]]
        scales = 4 * n * (-(-d // case["group"]) if case["group"] else 1)
        return {"bytes": n * d * (e * (3 if case["residual"] else 1) + out) + d * e +
                (scales if case["out"] == "i8" else 0), "flops": 6 * n * d}
    ff = case["ff"]
    if kind == "gated":
        n = case["n"]
        return {"bytes": 2 * (n * d + 2 * ff * d + n * ff * (3 if case["saved"] else 1)),
                "flops": 4 * n * d * ff}
    if kind == "gated_grad":
        n = case["n"]
        return {"bytes": 2 * (2 * n * d + 4 * ff * d + 3 * n * ff) +
                (2 * ff * d if case["masked"] else 0), "flops": 8 * n * d * ff}
    packed = ff * (d / 2 + 2 * -(-d // case["group"]))
    if kind == "w4_pack":
        return {"bytes": packed + ff * d * (2 if case["dtype"] == "bf16" else 4),
                "flops": 3 * ff * d}
    n, both = case["n"], 2 if kind == "w4_gated" else 1
    x = n * d * 2 if case["x"] == "bf16" else \
        n * (d + 4 * (-(-d // case["x_group"]) if case["x_group"] else 1))
    return {"bytes": both * packed + x + 2 * n * ff, "flops": 2 * both * n * d * ff}


def _exact_codes(Q, d):
    """Code of every weight, by index: where in its row value k is kept."""
    k = torch.arange(d, device=Q.device)
    chunk, within = k // 128, k % 128
    dword, block, code = within // 32, within % 32 // 8, within % 8
    nibble = code // 2 + 4 * (code % 2)
    byte = Q[:, chunk * 64 + block * 16 + dword * 4 + nibble // 2].long()
    return torch.where(nibble % 2 == 1, byte // 16, byte % 16) - 8


def exact(case, seed):
    st = prepare(case, seed)
    kind, d = case["kind"], case["d"]
    if kind == "norm":
        s = st["X"].double() + (0 if st["R"] is None else st["R"].double())
        S = s if st["R"] is not None else None
        y = s / (s.pow(2).sum(1, keepdim=True) / d + EPS).sqrt() * st["weight"].double()
        if case["out"] != "i8":
            return {"S": S, "Y": y, "scales": None}
        of = torch.arange(d, device=y.device) // (case["group"] or d)
        top = torch.zeros(case["n"], int(of[-1]) + 1, dtype=torch.float64, device=y.device)
        top.scatter_reduce_(1, of.expand(case["n"], d), y.abs(), "amax")
        each = (top / 127)[:, of]
        return {"S": S, "Y": torch.where(each > 0, (y / each).round() * each, 0.0),
                "scales": top / 127}
    if kind == "norm_grad":
        s, dy, w = st["S"].double(), st["dY"].double(), st["weight"].double()
        m = s.pow(2).sum(1, keepdim=True) / d + EPS
        # y = w s m^(-1/2), and dm/ds = 2 s / d
        dx = dy * w / m.sqrt() - s * (dy * w * s).sum(1, keepdim=True) / (d * m * m.sqrt())
        if st["dS"] is not None:
            dx += st["dS"].double()
        return {"dX": dx, "dweight": (dy * s / m.sqrt()).sum(0)}
    if kind == "gated":
        x = st["X"].double()
        g = torch.mm(x, st["Wg"].double().t().contiguous())
        u = torch.mm(x, st["Wu"].double().t().contiguous())
        return {"H": g * torch.sigmoid(g) * u, "G": g if case["saved"] else None,
                "U": u if case["saved"] else None}
    if kind == "gated_grad":
        g, sig = st["G"].double(), torch.sigmoid(st["G"].double())
        slope = sig + g * sig * (1 - sig)  # of g sigmoid(g)
        both = torch.cat([slope * st["U"].double() * st["dH"].double(),
                          sig * g * st["dH"].double()], 1)
        dx = torch.mm(both, torch.cat([st["Wg"], st["Wu"]]).double())
        dw = torch.mm(both.t().contiguous(), st["X"].double())
        if case["masked"]:
            dw = torch.where(torch.cat([st["mask_g"], st["mask_u"]]) != 0, dw, 0.0)
        return {"dX": dx, "dWg": dw[:case["ff"]], "dWu": dw[case["ff"]:]}
    if kind == "w4_pack":
        of = torch.arange(d, device="cuda") // case["group"]
        top = torch.zeros(case["ff"], int(of[-1]) + 1, dtype=torch.float64, device="cuda")
        top.scatter_reduce_(1, of.expand(case["ff"], d), st["W"].double().abs(), "amax")
        return {"Q": None, "scales": top / 7}
    x = st["X"].double()
    of = torch.arange(d, device=x.device)
    if st["x_scales"] is not None:
        x = x * st["x_scales"].double()[:, of // (case["x_group"] or d)]
    w = _exact_codes(st["Q"], d) * st["scales"].double()[:, of // case["group"]]
    y = torch.mm(x, w.t().contiguous())
    if kind == "w4_gated":
        w = _exact_codes(st["Q2"], d) * st["scales2"].double()[:, of // case["group"]]
        y = y * torch.sigmoid(y) * torch.mm(x, w.t().contiguous())
    return {"Y": y}
