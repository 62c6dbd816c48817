"""The operators around a boundary that a stage's training step and its serving
path need beside the boundary itself, as timed passes: the residual addition
with its RMS norm (16-bit and 8-bit output), that norm's backward pass, the
AdamW step over many tensors with states in 32 or 8 bits, and the gradient
norm with its clip factor over the same tensors.

Kinds of pass
  norm    h = x + res + b I (the residual stream, the decoder's skip), y = RMSNorm(h).
  norm8   the same with y in e4m3 and float32 scales per row or column group.
  back    gradient of x (and res) and of the gain.
  adamw   one optimizer step on a stage's tensors, float32 states.
  adamw8  the same with e4m3 states and a float32 scale per 256 elements.
  gnorm   the 2-norm of a stage's gradients and the clip factor.

A stage's tensors lie one after the other in one buffer per role, each from a
multiple of 256 elements on; what lies between them is zero and stays so.
"""
from __future__ import annotations

import math

import torch

own = False  # whether run() calls the framework's operators

EPS = 1e-5        # of the norm
BETAS = (0.9, 0.95)
ADAM_EPS = 1e-8
LR, DECAY, STEP = 1e-4, 0.1, 100
MAX_NORM = 1.0
BLOCK = 256       # elements per scale of an 8-bit state
E4M3_MAX = 448.0
E4M3_TINY = 2.0 ** -9
FLOOR = 2.0 ** -126


def listed():
    return [
        # serving: the next token of one sequence enters a stage
        {"name": "norm_token", "op": "norm", "T": 1, "n": 4096, "r": 32, "res": True},
        # training: the headline boundary's micro-batches (n4096_r32_t3)
        {"name": "norm_n4096", "op": "norm", "T": 16384, "n": 4096, "r": 32, "res": True},
        # serving with 8-bit products: a ragged batch of decoding sequences
        {"name": "norm8_ragged", "op": "norm8", "T": 77, "n": 2112, "r": 20, "res": True, "group": 64},
        # prefill at the 70B-class width (n8192_r64_lognormal), the largest norm
        {"name": "norm8_n8192", "op": "norm8", "T": 32768, "n": 8192, "r": 64, "res": True, "group": 128},
        # training backward, ragged tokens and width
        {"name": "back_ragged", "op": "back", "T": 3001, "n": 2112, "res": True, "acc": False},
        # training backward of the headline boundary's norm
        {"name": "back_n4096", "op": "back", "T": 16384, "n": 4096, "res": True, "acc": False},
        # the smallest configuration's boundary weights and gains (tiny_n512_r4)
        {"name": "adamw_tiny", "op": "adamw", "blocks": 0, "n": 512, "N": 0, "d_ff": 0, "r": 4, "g16": False},
        # a stage of one block at the benchmark's widths, the largest update
        {"name": "adamw_n4096", "op": "adamw", "blocks": 1, "n": 4096, "N": 6144, "d_ff": 14336, "r": 32, "g16": False},
        # eight small blocks of odd sizes
        {"name": "adamw8_ragged", "op": "adamw8", "blocks": 8, "n": 499, "N": 1497, "d_ff": 1733, "r": 20, "g16": False},
        # a stage of four blocks at the 1B-class width, gradients in 16 bits
        {"name": "adamw8_n2048", "op": "adamw8", "blocks": 4, "n": 2048, "N": 6144, "d_ff": 7168, "r": 16, "g16": True},
        # hundreds of small tensors
        {"name": "gnorm_many", "op": "gnorm", "blocks": 48, "n": 512, "N": 640, "d_ff": 1792, "r": 4, "g16": False},
        # the clip factor of the benchmark's widths
        {"name": "gnorm_n4096", "op": "gnorm", "blocks": 1, "n": 4096, "N": 6144, "d_ff": 14336, "r": 32, "g16": False},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm8", "norm8", "back", "back", "adamw", "adamw8", "gnorm"])
    if op in ("norm", "norm8", "back"):
        T = _log(rng, 1, 32768)
        n = _log(rng, 64, 8192, 8)
        case = {"op": op, "T": T, "n": n, "res": rng.random() < 0.8}
        if op == "back":
            case["acc"] = rng.random() < 0.4
        else:
            case["r"] = min(n, _log(rng, 4, 256, 4)) // 4 * 4 if rng.random() < 0.7 else 0
        if op == "norm8":
            case["group"] = rng.choice([0, 32, 64, 128, 256])
            if case["group"]:
                case["n"] = max(case["group"], n // case["group"] * case["group"])
        return case
    n = _log(rng, 32, 4096)
    case = {"op": op, "n": n, "N": rng.randrange(n, 3 * n), "d_ff": rng.randrange(n, 7 * n // 2),
            "r": max(4, n // 128 // 4 * 4), "g16": rng.random() < 0.4}
    each = _block_elements(case)
    case["blocks"] = _log(rng, 1, max(1, min(64, 200_000_000 // each)))
    return case


def _block_elements(case):
    n = case["n"]
    return n * case["N"] + n * n + 3 * n * case["d_ff"] + 2 * n


def _sizes(case):
    """Elements and decay of each tensor of a stage: its blocks' QKV, output, gate, up and down
    projections and two gains, then the boundary's W_e and W_d and the gains before them."""
    n, f, r = case["n"], case["d_ff"], case["r"]
    block = [(n * case["N"], True), (n * n, True), (n * f, True), (n * f, True), (f * n, True), (n, False), (n, False)]
    return block * case["blocks"] + [(n * r, True), (r * n, True), (n, False), (n, False)]


def _places(case):
    """(offset, elements, decay) of each tensor, and the buffers' length."""
    at, out = 0, []
    for k, d in _sizes(case):
        out.append((at, k, d))
        at += -(-k // BLOCK) * BLOCK
    return out, at


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * seed + 17)
    dev = torch.device("cuda")
    bf = torch.bfloat16

    def rn(*s, std=1.0):
        return torch.randn(*s, generator=g, device=dev) * std

    if case["op"] in ("norm", "norm8"):
        T, n, r = case["T"], case["n"], case["r"]
        tok = torch.exp(rn(T, 1, std=0.5))
        d = {"x": (rn(T, n) * tok).to(bf), "gamma": 1.0 + rn(n, std=0.1)}
        d["res"] = (rn(T, n) * tok).to(bf) if case["res"] else None
        d["b"] = rn(T, r).to(bf) if r else None
        d["h"] = torch.empty(T, n, dtype=bf, device=dev)
        if case["op"] == "norm":
            d["y"] = torch.empty(T, n, dtype=bf, device=dev)
            d["rstd"] = torch.empty(T, dtype=torch.float32, device=dev)
        else:
            d["y"] = torch.empty(T, n, dtype=torch.float8_e4m3fn, device=dev)
            d["scale"] = torch.empty(T, n // (case["group"] or n), dtype=torch.float32, device=dev)
        return d
    if case["op"] == "back":
        T, n = case["T"], case["n"]
        tok = torch.exp(rn(T, 1, std=0.5))
        h = (rn(T, n) * tok).to(bf)
        rstd = (1.0 / torch.sqrt((h.double() ** 2).mean(1) + EPS)).float()
        return {"h": h, "rstd": rstd, "gamma": 1.0 + rn(n, std=0.1), "g_y": rn(T, n, std=0.1).to(bf),
                "g_h": rn(T, n, std=0.1).to(bf) if case["res"] else None,
                "g_x": torch.empty(T, n, dtype=bf, device=dev), "dgamma": rn(n) if case["acc"] else torch.empty(n, device=dev)}
    places, size = _places(case)
    # each tensor's own gradient size, as depths and kinds of layers have them
    count = torch.tensor([-(-k // BLOCK) for _, k, _ in places], device=dev)
    sigma = torch.exp(rn(len(places)) - 6.0).repeat_interleave(count)[:, None]
    live = torch.ones(size, device=dev, dtype=torch.bool)
    for at, k, _ in places:
        live[at + k:at + -(-k // BLOCK) * BLOCK] = False
    live = live.view(-1, BLOCK)
    grad = rn(size // BLOCK, BLOCK) * sigma * live
    d = {"g": (grad.to(bf) if case["g16"] else grad).view(-1), "places": places}
    if case["op"] == "gnorm":
        d["out"] = torch.empty(2, device=dev)
        return d
    gain = torch.tensor([0.0 if k else 1.0 for _, _, k in places], device=dev).repeat_interleave(count)[:, None]
    d["p"] = ((gain + rn(size // BLOCK, BLOCK, std=0.02)) * live).view(-1)
    d["copy"] = d["p"].to(bf)
    d["wd"] = torch.tensor([DECAY if k else 0.0 for _, _, k in places], device=dev).repeat_interleave(count)[:, None]
    m = rn(size // BLOCK, BLOCK, std=0.3) * sigma * live
    v = (sigma * (0.3 + torch.rand(size // BLOCK, BLOCK, generator=g, device=dev))) ** 2 * live
    if case["op"] == "adamw":
        d["m"], d["v"] = m.view(-1), v.view(-1)
    else:
        for name, t in (("m", m), ("u", torch.sqrt(v))):
            s = (t.abs().amax(1, keepdim=True) / E4M3_MAX).clamp(min=FLOOR)
            d[name], d[name + "_scale"] = (t / s).to(torch.float8_e4m3fn).view(-1), s.view(-1)
    return d


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2604_11947_amd import resbm as R

        s["lib"] = lib = R.library()
        if case["op"] == "back":
            s["ws"] = lib.norm_workspace(case["T"], case["n"], "cuda")
        elif case["op"] in ("adamw", "adamw8", "gnorm"):
            s["plan"] = _plan(lib, case, s)
            if case["op"] == "gnorm":
                s["ws"] = lib.grad_norm_workspace(s["plan"])
    return s


def _plan(lib, case, s):
    """The list of tensors that a training program makes once: views of the buffers."""
    def views(t, scales=False):
        if scales:
            return [t[at // BLOCK:at // BLOCK + -(-k // BLOCK)] for at, k, _ in s["places"]]
        return [t[at:at + k] for at, k, _ in s["places"]]

    if case["op"] == "gnorm":
        return lib.grad_plan(views(s["g"]))
    more = {}
    if case["op"] == "adamw8":
        more = {"m_scale": views(s["m_scale"], True), "v_scale": views(s["u_scale"], True)}
    return lib.adamw_plan(views(s["p"]), views(s["g"]), views(s["m"]), views(s["v"] if case["op"] == "adamw" else s["u"]),
                          copy=views(s["copy"]), weight_decay=[DECAY if d else 0.0 for _, _, d in s["places"]], **more)


def run(s):
    return (_own_run if own else _plain_run)(s)


def _own_run(s):
    lib, op = s["lib"], s["case"]["op"]
    if op == "norm":
        lib.skip_norm_fwd(s["x"], s["gamma"], s["y"], res=s["res"], b=s["b"], h=s["h"], rstd=s["rstd"], eps=EPS)
        return [s["h"], s["y"], s["rstd"]]
    if op == "norm8":
        lib.skip_norm_q8_fwd(s["x"], s["gamma"], s["y"], s["scale"], res=s["res"], b=s["b"], h=s["h"], eps=EPS)
        return [s["h"], s["y"], s["scale"]]
    if op == "back":
        lib.skip_norm_bwd(s["h"], s["gamma"], s["rstd"], s["g_y"], s["g_x"], s["dgamma"], g_h=s["g_h"],
                          accumulate=s["case"]["acc"], ws=s["ws"])
        return [s["g_x"], s["dgamma"]]
    if op == "gnorm":
        lib.grad_norm(s["plan"], MAX_NORM, s["out"], ws=s["ws"])
        return s["out"]
    lib.adamw_update(s["plan"], LR, STEP, betas=BETAS, eps=ADAM_EPS)
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return [s[k] for k in ("p", "copy", "m", "v", "u", "m_scale", "u_scale") if k in s]


def _plain_norm(s):
    x = s["x"].float()
    if s["res"] is not None:
        x = x + s["res"].float()
    if s["b"] is not None:
        x[:, :s["b"].shape[1]] += s["b"].float()
    h = x.to(torch.bfloat16)
    x = h.float()
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return h, x * rstd * s["gamma"], rstd[:, 0]


def _plain_run(s):
    case = s["case"]
    op = case["op"]
    if op == "norm":
        h, y, rstd = _plain_norm(s)
        return [h, y.to(torch.bfloat16), rstd]
    if op == "norm8":
        h, y, _ = _plain_norm(s)
        T, n = y.shape
        y = y.view(T, -1, case["group"] or n)
        scale = (y.abs().amax(2, keepdim=True) / E4M3_MAX).clamp(min=FLOOR)
        return [h, (y * (1.0 / scale)).to(torch.float8_e4m3fn).view(T, n), scale[:, :, 0]]
    if op == "back":
        xhat = s["h"].float() * s["rstd"][:, None]
        gy = s["g_y"].float()
        w = gy * s["gamma"]
        g = (w - xhat * (w * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
        if s["g_h"] is not None:
            g = g + s["g_h"].float()
        dgamma = (gy * xhat).sum(0)
        s["dgamma"].copy_(dgamma + s["dgamma"] if case["acc"] else dgamma)
        return [g.to(torch.bfloat16), s["dgamma"]]
    if op == "gnorm":
        norm = torch.sqrt((s["g"].double() ** 2).sum())
        return torch.stack([norm, (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)]).float()
    b1, b2 = BETAS
    c1, c2 = 1.0 - b1 ** STEP, 1.0 - b2 ** STEP
    p, g = s["p"].view(-1, BLOCK), s["g"].view(-1, BLOCK).float()
    if op == "adamw":
        m, v = s["m"].view(-1, BLOCK), s["v"].view(-1, BLOCK)
    else:
        m = s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]
        v = (s["u"].float().view(-1, BLOCK) * s["u_scale"][:, None]) ** 2
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + g * (1.0 - b2) * g
    u = torch.sqrt(v)
    new = p * (1.0 - s["wd"].double() * LR).float() - m / (u * (1.0 / math.sqrt(c2)) + ADAM_EPS) * (LR / c1)
    s["p"].copy_(new.view(-1))
    s["copy"].copy_(s["p"])
    if op == "adamw":
        s["m"].copy_(m.view(-1))
        s["v"].copy_(v.view(-1))
        return _adamw_outputs(s)
    scale = (m.abs().amax(1, keepdim=True) / E4M3_MAX).clamp(min=FLOOR)
    s["m"].copy_((m * (1.0 / scale)).to(torch.float8_e4m3fn).view(-1))
    s["m_scale"].copy_(scale[:, 0])
    scale = (u.amax(1, keepdim=True) / E4M3_MAX).clamp(min=FLOOR)
    t = u * (1.0 / scale)
    s["u"].copy_(torch.where(u > 0, t.clamp(min=E4M3_TINY), t).to(torch.float8_e4m3fn).view(-1))
    s["u_scale"].copy_(scale[:, 0])
    return _adamw_outputs(s)


def work(case):
    op = case["op"]
    if op in ("norm", "norm8", "back"):
        T, n = case["T"], case["n"]
        if op == "back":
            each = 6 + 2 * case["res"]
            return {"bytes": T * (each * n + 4) + n * (8 + 4 * case["acc"]), "flops": T * n * (9 + case["res"])}
        each = 4 + 2 * case["res"] + (2 if op == "norm" else 1)
        scales = 1 if op == "norm" else n // (case["group"] or n)
        return {"bytes": T * (each * n + 2 * case["r"] + 4 * scales) + 4 * n,
                "flops": T * (n * (4 + case["res"] + 2 * (op == "norm8")) + case["r"])}
    k = sum(k for k, _ in _sizes(case))
    g = 2 if case["g16"] else 4
    if op == "gnorm":
        return {"bytes": k * g + 8, "flops": 2 * k}
    if op == "adamw":
        return {"bytes": k * (g + 8 + 16 + 2), "flops": 14 * k}
    return {"bytes": k * (g + 8 + 4 + 2) + 16 * sum(-(-e // BLOCK) for e, _ in _sizes(case)), "flops": 22 * k}


def exact(case, seed):
    """The definitions in 64 bits: h rounded once to bf16, since y is defined on the stream as it is stored;
    8-bit values before their rounding."""
    s = _inputs(case, seed)
    f = torch.float64
    if case["op"] in ("norm", "norm8"):
        T, n = s["x"].shape
        h = s["x"].to(f)
        if s["res"] is not None:
            h = h.add_(s["res"])
        if s["b"] is not None:
            h[:, :case["r"]].add_(s["b"])
        hs = h.to(torch.bfloat16).to(f)
        rstd = hs.square().sum(1).div_(n).add_(EPS).rsqrt_()
        y = hs.mul_(rstd[:, None]).mul_(s["gamma"].to(f))
        if case["op"] == "norm":
            return [h, y, rstd]
        y = y.view(T, -1, case["group"] or n)
        scale = y.abs().max(2).values.div_(E4M3_MAX).clamp_(min=FLOOR)
        return [h, y.div_(scale[:, :, None]).view(T, n), scale]
    if case["op"] == "back":
        n = case["n"]
        a = s["rstd"].to(f)[:, None]
        xhat = s["h"].to(f).mul_(a)
        gy = s["g_y"].to(f)
        dgamma = (gy * xhat).sum(0)
        if case["acc"]:
            dgamma += s["dgamma"]
        w = gy.mul_(s["gamma"].to(f))
        c = (w * xhat).sum(1, keepdim=True) / n
        g = w.sub_(xhat.mul_(c)).mul_(a)
        return [g if s["g_h"] is None else g.add_(s["g_h"]), dgamma]
    g = s["g"].to(f)
    if case["op"] == "gnorm":
        norm = float(torch.dot(g, g)) ** 0.5
        return torch.tensor([norm, min(1.0, MAX_NORM / (norm + 1e-6))], dtype=f)
    b1, b2 = BETAS
    if case["op"] == "adamw":
        m, v = s["m"].to(f), s["v"].to(f)
    else:
        m = s["m"].to(f) * s["m_scale"].to(f).repeat_interleave(BLOCK)
        v = (s["u"].to(f) * s["u_scale"].to(f).repeat_interleave(BLOCK)).square_()
    m = m.mul_(b1).add_(g, alpha=1.0 - b1)
    v = v.mul_(b2).addcmul_(g, g, value=1.0 - b2)
    u = v.sqrt()
    step = (m / (1.0 - b1 ** STEP)).div_((u / math.sqrt(1.0 - b2 ** STEP)).add_(ADAM_EPS))
    p = s["p"].to(f)
    p = p - LR * (step + s["wd"].to(f).expand(-1, BLOCK).reshape(-1) * p)
    if case["op"] == "adamw":
        return [p, p, m, v]
    out = [p, p]
    scales = []
    for t in (m, u):
        t = t.view(-1, BLOCK)
        sc = t.abs().max(1).values.div_(E4M3_MAX).clamp_(min=FLOOR)
        out.append((t / sc[:, None]).view(-1))
        scales.append(sc)
    return out + scales
