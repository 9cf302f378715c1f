"""The operators around a pruned linear layer that a language model's step needs, and the calls their speed is judged by.

  logprobs   sdgp_token_logprobs (+ _bwd): log probabilities of given tokens, entropy and top alternatives of every row of
             logits; its gradient is the dL/dO that the last linear layer's pruned backward pass starts from
  norm       sdgp_block_norm (+ _bwd): the norm after a block, its gate, the scaled residual and the norm before the next block
  adamw      optim.AdamW.step: one step over all tensors, fp32 states or states in 8 bits, with the bf16 copies that the
             layers multiply with

``run`` computes each either in plain torch, 32 bits throughout and rounded once at the end (``own`` false), or with this
library's kernels (``own`` true).  ``exact`` is the definition in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_BLOCK = 256          # elements that share a scale in an 8-bit state
_BETAS, _EPS, _DECAY = (0.9, 0.999), 1e-8, 0.01


# ------------------------------------------------------------------------------------------------------------- cases

def _logprobs(name, rows, V, dtype, mode, top, scale=1.0, pad=0, banned=0.0):
    c = {"op": "logprobs", "rows": rows, "V": V, "dtype": dtype, "mode": mode, "top": top, "scale": scale, "pad": pad,
         "banned": banned}
    return dict(c, name=name) if name else c


def _norm(name, rows, D, dtype, mode, gate, groups, block=True, wdtype="f32", residual_scale=1.0):
    c = {"op": "norm", "rows": rows, "D": D, "dtype": dtype, "mode": mode, "gate": gate, "groups": groups, "block": block,
         "wdtype": wdtype, "residual_scale": residual_scale}
    return dict(c, name=name) if name else c


def _adamw(name, net, bits, param, grad, copies, count=0, lo=0, hi=0, shape_seed=0):
    c = {"op": "adamw", "net": net, "bits": bits, "param": param, "grad": grad, "copies": copies, "count": count, "lo": lo,
         "hi": hi, "shape_seed": shape_seed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: the next token of four sequences, its eight best alternatives; few rows over a long vocabulary
        _logprobs("logp_decode_4x131072", 4, 131072, "bf16", "fwd", 8, scale=1.25),
        # the classifier of the repository's ResNet-50 at batch 256, forward and gradient; its launches are most of it
        _logprobs("logp_classifier_256x1000", 256, 1000, "f32", "train", 5),
        # policy-gradient training over an odd vocabulary cut out of padded logits, some tokens not allowed
        _logprobs("logp_policy_2048x50021", 2048, 50021, "bf16", "train", 4, scale=0.8, pad=155, banned=0.02),
        # pre-training: a batch's tokens, no alternatives asked for
        _logprobs("logp_train_8192x65536", 8192, 65536, "bf16", "train", 0),
        # serving: one token through a block's norms
        _norm("norm_token_1x2048", 1, 2048, "bf16", "fwd", "channel", 1),
        # odd width in fp32, a gate value for every element
        _norm("norm_f32_4099x1001", 4099, 1001, "f32", "train", "row", 4099, residual_scale=0.5),
        # a gate for each of 16 samples of 1024 tokens, as conditioned blocks have it
        _norm("norm_sample_16384x2048", 16384, 2048, "bf16", "train", "sample", 16, wdtype="bf16"),
        # the largest: a wide model's training batch
        _norm("norm_wide_32768x4096", 32768, 4096, "bf16", "train", "channel", 1),
        # the repository's small linear layer: one tensor, the call is most of it
        _adamw("adamw32_linear_128x256", "linear", 32, "f32", "f32", False),
        # all 161 tensors of ResNet-50, fp32 states, bf16 copies for the kernels that multiply
        _adamw("adamw32_resnet50", "resnet50", 32, "f32", "f32", True),
        # the same with states in 8 bits
        _adamw("adamw8_resnet50", "resnet50", 8, "f32", "f32", True),
        # the matrices of a larger model, 8-bit states, gradients in bf16
        _adamw("adamw8_matrices_24x8388608", "drawn", 8, "f32", "bf16", True, 24, 8388608, 8388608, 1),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "norm", "adamw"])
    if op == "logprobs":
        V = _spread(rng, 10, 131072)
        rows = _spread(rng, 1, max(1, min(16384, 8192 * 65536 // V // 2)))
        return _logprobs(None, rows, V, rng.choice(["f32", "bf16"]), rng.choice(["fwd", "train"]),
                         min(V, rng.choice([0, 1, 4, 8, 20, 64])), scale=rng.choice([0.5, 0.8, 1.0, 1.0, 1.5]),
                         pad=rng.choice([0, 0, 1, 24, 128]), banned=rng.choice([0.0, 0.0, 0.05, 0.5]))
    if op == "norm":
        D = _spread(rng, 16, 8192)
        gate = rng.choice(["none", "channel", "sample", "row"])
        groups = _spread(rng, 2, 64) if gate == "sample" else 1
        rows = _spread(rng, 1, max(1, 32768 * 4096 // D // 2 // groups)) * groups
        rows = max(groups, min(rows, 65536 // groups * groups))
        return _norm(None, rows, D, rng.choice(["f32", "bf16", "bf16"]), rng.choice(["fwd", "train"]), gate,
                     {"none": 0, "channel": 1, "sample": groups, "row": rows}[gate], block=gate != "none" or rng.random() < 0.5,
                     wdtype=rng.choice(["f32", "same"]), residual_scale=rng.choice([1.0, 0.7]))
    count = _spread(rng, 1, 200)
    hi = _spread(rng, 100, min(16777216, 24 * 8388608 // count))
    param = rng.choice(["f32", "bf16"])
    return _adamw(None, "drawn", rng.choice([32, 8]), param, rng.choice(["f32", "bf16"]), param == "f32" and rng.random() < 0.5,
                  count, max(1, hi // rng.choice([1, 30, 1000])), hi, rng.randrange(1 << 30))


# ------------------------------------------------------------------------------------------------------------ inputs

def _resnet50_shapes():
    """161 tensors: 53 convolutions [out, R, S, in], two vectors for the norm behind each, the classifier and its bias."""
    convs, prev = [(64, 7, 7, 3)], 64
    for stage, (width, blocks) in enumerate(((64, 3), (128, 4), (256, 6), (512, 3))):
        for blk in range(blocks):
            convs += [(width, 1, 1, prev), (width, 3, 3, width), (4 * width, 1, 1, width)]
            if blk == 0:
                convs.append((4 * width, 1, 1, prev))
            prev = 4 * width
    shapes = []
    for c in convs:
        shapes += [c, (c[0],), (c[0],)]
    return shapes + [(1000, 2048), (1000,)]


def _shapes(case):
    if case["net"] == "linear":
        return [(128, 256)]
    if case["net"] == "resnet50":
        return _resnet50_shapes()
    rng = random.Random(case["shape_seed"])
    return [(_spread(rng, case["lo"], case["hi"]),) for _ in range(case["count"])]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 13)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _prepare_logprobs(case, g):
    rows, V = case["rows"], case["V"]
    wide = _randn(g, rows, V + case["pad"]) * 2.5
    tokens = torch.randint(0, V, (rows,), device="cuda", generator=g)
    sure = torch.rand(rows, device="cuda", generator=g) * 12          # how clearly the model prefers the given token
    wide.scatter_add_(1, tokens[:, None], sure[:, None])
    if case["banned"]:
        wide.masked_fill_(torch.rand(rows, V + case["pad"], device="cuda", generator=g) < case["banned"], -math.inf)
        wide.scatter_(1, tokens[:, None], sure[:, None])               # a token that was sampled was allowed
    tokens = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.05, -100, tokens)   # prompt tokens: no loss
    state = {"logits": wide.to(_DT[case["dtype"]])[:, :V], "tokens": tokens, "top": case["top"], "scale": case["scale"]}
    if case["mode"] == "train":
        state["g_logp"] = -torch.rand(rows, device="cuda", generator=g) / rows
        state["g_entropy"] = torch.full((rows,), -0.01 / rows, device="cuda") * torch.rand(rows, device="cuda", generator=g)
    return state


def _prepare_norm(case, g):
    rows, D, dt = case["rows"], case["D"], _DT[case["dtype"]]
    wdt = dt if case["wdtype"] == "same" else _DT[case["wdtype"]]
    state = {"x": (_randn(g, rows, D) * 2).to(dt), "w_pre": (1 + 0.2 * _randn(g, D)).to(wdt), "u": None, "gate": None,
             "w_post": None, "residual_scale": case["residual_scale"], "groups": case["groups"]}
    if case["block"]:
        state["u"] = (_randn(g, rows, D) * (0.1 + torch.rand(D, device="cuda", generator=g))).to(dt)
        state["w_post"] = (1 + 0.2 * _randn(g, D)).to(wdt)
        if case["gate"] != "none":
            state["gate"] = (_randn(g, case["groups"], D) * 0.5).to(dt)
    if case["mode"] == "train":
        state["dy"] = (_randn(g, rows, D) * 1e-3).to(dt)
        state["dh"] = (_randn(g, rows, D) * 1e-3).to(dt)
    return state


def _prepare_adamw(case, g):
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + -(-n // _BLOCK) * _BLOCK)
    total = starts[-1]
    state = {"shapes": shapes, "sizes": sizes, "starts": starts[:-1], "bits": case["bits"], "steps": 40, "seed": 1234}
    dt = _DT[case["param"]]
    inside = torch.zeros(total, device="cuda", dtype=torch.bool)
    for s, n in zip(starts, sizes):
        inside[s:s + n] = True
    # parameters of about 0.03, gradients of a few orders of magnitude, states as after some steps with such gradients
    level = torch.exp(_randn(g, total // _BLOCK) - 7).repeat_interleave(_BLOCK)
    state["params"] = (_randn(g, total) * 0.03 * inside).to(dt)
    grad = _randn(g, total) * level * inside
    avg = _randn(g, total) * level * 0.3 * inside
    rms = level * (0.5 + torch.rand(total, device="cuda", generator=g)) * inside
    gdt = _DT[case["grad"]]
    state["grads"] = [grad[s:s + n].to(gdt).reshape(shape) for s, n, shape in zip(starts, sizes, shapes)]
    if case["bits"] == 32:
        state["exp_avg"], state["exp_avg_sq"] = avg, rms * rms
    else:
        for key, x in (("exp_avg", avg), ("exp_avg_sq", rms)):
            top = x.view(-1, _BLOCK).abs().amax(1)
            scale = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 440.0)))
            state[key] = (x.view(-1, _BLOCK) / scale[:, None]).to(torch.float8_e4m3fn).reshape(-1)
            state[key + "_scale"] = scale
    if case["copies"]:
        state["copies"] = state["params"].to(torch.bfloat16)
    state["grad_scale"] = torch.full((1,), 0.75, device="cuda")          # as clipping by the global norm leaves it
    state["lr"] = 1e-3
    return state


def prepare(case, seed):
    g = _generator(seed)
    return {"op": case["op"], **{"logprobs": _prepare_logprobs, "norm": _prepare_norm, "adamw": _prepare_adamw}[case["op"]](case, g)}


# ------------------------------------------------------------------------------------------------------- plain forms

def _plain_logprobs(s):
    x = s["logits"].float()
    z = x * s["scale"]
    z -= z.amax(1, keepdim=True)
    e = torch.exp(z)
    total = e.sum(1, keepdim=True)
    p = e / total
    logq = z - torch.log(total)
    held = torch.where(p > 0, logq, 0.0)                                 # 0 log 0 = 0
    entropy = -(p * held).sum(1)
    given = s["tokens"] >= 0
    at = s["tokens"].clamp(min=0)[:, None]
    out = {"logp": torch.where(given, logq.gather(1, at)[:, 0], 0.0), "entropy": entropy}
    if s["top"]:
        left, ids, best = x.clone(), [], []
        for _ in range(s["top"]):
            i = left.argmax(1, keepdim=True)                             # the first of equal ones
            there = left.gather(1, i) > -math.inf
            ids.append(torch.where(there, i, -1))
            best.append(torch.where(there, logq.gather(1, i), -math.inf))
            left.scatter_(1, i, -math.inf)
        out["top_ids"], out["top_logp"] = torch.cat(ids, 1), torch.cat(best, 1)
    if "g_logp" in s:
        g, h = torch.where(given, s["g_logp"], 0.0)[:, None], s["g_entropy"][:, None]
        d = -p * (g + h * (held + entropy[:, None]))
        d.scatter_add_(1, at, g)
        out["dlogits"] = (d * s["scale"]).to(s["logits"].dtype)
    return out


def _plain_norm(s, eps=1e-6):
    x, w_pre = s["x"].float(), s["w_pre"].float()
    rows, D = x.shape
    y = x
    if s["u"] is not None:
        u, w_post = s["u"].float(), s["w_post"].float()
        r_u = torch.rsqrt((u * u).mean(1, keepdim=True) + eps)
        a = u * r_u
        gate = s["gate"].float().repeat_interleave(rows // s["groups"], 0) if s["gate"] is not None else torch.ones_like(w_post)
        y = s["residual_scale"] * x + gate * (a * w_post)
    dt = s["x"].dtype
    y = y.to(dt)
    yf = y.float()                                                       # what the next block and the gradient see
    r_y = torch.rsqrt((yf * yf).mean(1, keepdim=True) + eps)
    t = yf * r_y
    out = {"y": y, "h": (t * w_pre).to(dt)}
    if "dy" not in s:
        return out
    dh = s["dh"].float()
    dn = dh * w_pre
    dY = s["dy"].float() + r_y * (dn - t * (dn * t).mean(1, keepdim=True))
    out["dw_pre"] = (dh * t).sum(0)
    if s["u"] is None:
        return dict(out, dx=dY.to(dt))
    out["dx"] = (s["residual_scale"] * dY).to(dt)
    out["dw_post"] = (dY * gate * a).sum(0)
    if s["gate"] is not None:
        out["dgate"] = (dY * a * w_post).view(s["groups"], rows // s["groups"], D).sum(1).to(dt)
    da = dY * gate * w_post
    out["du"] = (r_u * (da - a * (da * a).mean(1, keepdim=True))).to(dt)
    return out


def _mix(seed, e):
    """The library's 32-bit counter hash of (seed, element), one word an element."""
    mask = 0xFFFFFFFF
    v = (0xA54FF53A ^ ((seed & mask) * 0x9E3779B9 & mask) ^ ((seed >> 32) * 0x510E527F & mask)) ^ (e & mask) ^ ((e >> 32) * 0xBB67AE85 & mask)
    v = v ^ (v >> 16)
    v = v * 0x6A09E667 & mask
    v = v ^ (v >> 15)
    v = v * 0xBB67AE85 & mask
    return v ^ (v >> 16)


def _to_8bit(x, u, keep):
    """x as e4m3 codes under one power of two for each block, rounded up with the probability of what is cut off (u in
    [0, 1) decides); ``keep``: what is not zero is not stored as zero."""
    b = x.view(-1, _BLOCK)
    f, e = torch.frexp(b.abs().amax(1))
    power = torch.where(f > 0, (e - 9 + (f > 0.875)).clamp(min=-126), 0)
    scale = torch.ldexp(torch.ones_like(f), power)
    y = (b * torch.ldexp(torch.ones_like(f), -power)[:, None]).view(-1)
    _, e = torch.frexp(y)
    e = torch.where(y != 0, e - 1, -6).clamp(min=-6)                     # below 2^-6 the codes are evenly spaced
    c = torch.floor(torch.ldexp(y.abs(), 3 - e) + u)
    if keep:
        c = torch.where((y != 0) & (c == 0), 1.0, c)
    return torch.copysign(torch.ldexp(c, e - 3), y).to(torch.float8_e4m3fn), scale


def _plain_adamw(s):
    (b1, b2), t = _BETAS, s["steps"] + 1
    s["steps"] = t
    p = s["params"].float()
    g = torch.zeros_like(p)
    torch._foreach_copy_([g[i:i + n] for i, n in zip(s["starts"], s["sizes"])], [x.reshape(-1) for x in s["grads"]])
    g *= s["grad_scale"]
    if s["bits"] == 32:
        m, v = s["exp_avg"], s["exp_avg_sq"]
    else:
        m = (s["exp_avg"].float().view(-1, _BLOCK) * s["exp_avg_scale"][:, None]).view(-1)
        r = (s["exp_avg_sq"].float().view(-1, _BLOCK) * s["exp_avg_sq_scale"][:, None]).view(-1)
        v = r * r
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    r = torch.sqrt(v)
    p = p * (1 - s["lr"] * _DECAY) - (s["lr"] / (1 - b1 ** t)) * (m / (r / math.sqrt(1 - b2 ** t) + _EPS))
    s["params"].copy_(p)
    out = {"params": s["params"], "exp_avg": s["exp_avg"], "exp_avg_sq": s["exp_avg_sq"]}
    if s["bits"] == 32:
        s["exp_avg"].copy_(m)
        s["exp_avg_sq"].copy_(v)
    else:
        h = _mix(s["seed"] + t, torch.arange(p.numel(), device=p.device))
        for key, x, u, keep in (("exp_avg", m, h & 0xFFFF, False), ("exp_avg_sq", r, h >> 16, True)):
            code, scale = _to_8bit(x, u.float() / 65536, keep)
            s[key].copy_(code)
            s[key + "_scale"].copy_(scale)
            out[key + "_scale"] = s[key + "_scale"]
    if "copies" in s:
        s["copies"].copy_(p)
        out["copies"] = s["copies"]
    return out


# ---------------------------------------------------------------------------------------------- the library's kernels

def _own_logprobs(s):
    import paper_2202_00774_amd as sdgp
    logp, entropy, top_logp, top_ids, stats = sdgp.sdgp_token_logprobs(s["logits"], s["tokens"], top=s["top"], scale=s["scale"])
    out = {"logp": logp, "entropy": entropy}
    if s["top"]:
        out["top_ids"], out["top_logp"] = top_ids, top_logp
    if "g_logp" in s:
        out["dlogits"] = sdgp.sdgp_token_logprobs_bwd(s["logits"], s["tokens"], stats, entropy, s["g_logp"], s["g_entropy"],
                                                      scale=s["scale"])
    return out


def _own_norm(s):
    import paper_2202_00774_amd as sdgp
    y, h, stats = sdgp.sdgp_block_norm(s["x"], s["u"], s["gate"], s["w_post"], s["w_pre"], residual_scale=s["residual_scale"])
    out = {"y": y, "h": h}
    if "dy" in s:
        dx, du, dgate, dw_post, dw_pre = sdgp.sdgp_block_norm_bwd(s["dy"], s["dh"], y, stats, s["u"], s["gate"], s["w_post"],
                                                                  s["w_pre"], residual_scale=s["residual_scale"])
        out.update({k: v for k, v in (("dx", dx), ("du", du), ("dgate", dgate), ("dw_post", dw_post), ("dw_pre", dw_pre)) if v is not None})
    return out


def _own_adamw(s):
    if "optimizer" not in s:
        # made once, in front of the training loop
        from paper_2202_00774_amd.optim import AdamW
        views = lambda flat: [flat[i:i + n].view(shape) for i, n, shape in zip(s["starts"], s["sizes"], s["shapes"])]  # noqa: E731
        blocks = lambda flat: [flat[i // _BLOCK:-(-(i + n) // _BLOCK)] for i, n in zip(s["starts"], s["sizes"])]  # noqa: E731
        state = {k: views(s[k]) for k in ("exp_avg", "exp_avg_sq")}
        if s["bits"] == 8:
            state.update({k: blocks(s[k]) for k in ("exp_avg_scale", "exp_avg_sq_scale")})
        s["optimizer"] = AdamW(views(s["params"]), lr=s["lr"], betas=_BETAS, eps=_EPS, weight_decay=_DECAY, state_bits=s["bits"],
                               copies=views(s["copies"]) if "copies" in s else None, seed=s["seed"], state=state, steps=s["steps"])
    s["optimizer"].step(s["grads"], grad_scale=s["grad_scale"])
    return {k: s[k] for k in ("params", "exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale", "copies") if k in s}


def run(state):
    if own:
        return {"logprobs": _own_logprobs, "norm": _own_norm, "adamw": _own_adamw}[state["op"]](state)
    return {"logprobs": _plain_logprobs, "norm": _plain_norm, "adamw": _plain_adamw}[state["op"]](state)


# -------------------------------------------------------------------------------------------------------------- work

def work(case):
    if case["op"] == "logprobs":
        n, train = case["rows"] * case["V"], case["mode"] == "train"
        return {"bytes": n * _SIZE[case["dtype"]] * (2 if train else 1) + case["rows"] * (24 + 12 * case["top"]),
                "flops": n * (14 if train else 6)}
    if case["op"] == "norm":
        n, train = case["rows"] * case["D"], case["mode"] == "train"
        tensors = (8 if train else 4) if case["block"] else (5 if train else 2)   # x u | y h | dy dh | dx du
        gates = case["groups"] * case["D"] * (2 if train else 1)
        return {"bytes": (n * tensors + gates) * _SIZE[case["dtype"]] + case["D"] * (12 if train else 8), "flops": n * (30 if train else 10)}
    n = sum(math.prod(s) for s in _shapes(case))
    each = 2 * _SIZE[case["param"]] + _SIZE[case["grad"]] + (2 if case["copies"] else 0) + (16 if case["bits"] == 32 else 4 + 16 / _BLOCK)
    return {"bytes": n * each, "flops": n * 15}


# ------------------------------------------------------------------------------------------------------------- exact

def _exact_logprobs(s):
    rows = s["logits"].shape[0]
    parts = []
    step = max(1, (1 << 27) // s["logits"].shape[1])
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        z = s["logits"][lo:hi].double() * s["scale"]
        lse = torch.logsumexp(z, 1)
        logq = z - lse[:, None]
        q = logq.exp()
        tokens = s["tokens"][lo:hi]
        entropy = torch.special.entr(q).sum(1)
        chosen = logq[torch.arange(hi - lo, device=z.device), tokens.clamp(min=0)]
        part = {"logp": chosen.where(tokens >= 0, torch.zeros_like(chosen)), "entropy": entropy}
        if s["top"]:
            part["top_logp"] = logq.topk(s["top"], 1).values
        if "g_logp" in s:
            g, h = s["g_logp"][lo:hi].double() * (tokens >= 0), s["g_entropy"][lo:hi].double()
            d = -q * g[:, None] - h[:, None] * torch.where(q > 0, q * (logq + entropy[:, None]), torch.zeros_like(q))
            d[torch.arange(hi - lo, device=z.device), tokens.clamp(min=0)] += g
            part["dlogits"] = d * s["scale"]
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    return dict(out, top_ids=None) if s["top"] else out


def _exact_norm(s, eps=1e-6):
    """The stored y is rounded: h and the gradients are those of the values that are stored."""
    sums, whole = {}, {k: [] for k in ("y", "h", "dx", "du")}
    rows, D = s["x"].shape
    gate = None if s["gate"] is None else s["gate"].double()
    w_pre = s["w_pre"].double()
    w_post = None if s["w_post"] is None else s["w_post"].double()
    per = rows // s["groups"] if gate is not None else rows
    dgate = torch.zeros(gate.shape, dtype=torch.float64, device="cuda") if gate is not None else None
    step = max(1, (1 << 25) // D)
    for lo in range(0, rows, step):
        hi = min(rows, lo + step)
        group = torch.arange(lo, hi, device="cuda") // per
        x = s["x"][lo:hi].double()
        y = x
        if s["u"] is not None:
            u = s["u"][lo:hi].double()
            size = torch.sqrt(u.square().mean(1, keepdim=True) + eps)
            a = u / size
            k = gate[group] if gate is not None else torch.ones_like(a)
            y = s["residual_scale"] * x + k * a * w_post
        whole["y"].append(y)
        y = y.to(s["x"].dtype).double()
        ysize = torch.sqrt(y.square().mean(1, keepdim=True) + eps)
        n = y / ysize
        whole["h"].append(n * w_pre)
        if "dy" not in s:
            continue
        dh = s["dh"][lo:hi].double()
        q = dh * w_pre
        back = s["dy"][lo:hi].double() + (q - n * (q * n).sum(1, keepdim=True) / D) / ysize
        sums["dw_pre"] = sums.get("dw_pre", 0) + (dh * n).sum(0)
        if s["u"] is None:
            whole["dx"].append(back)
            continue
        whole["dx"].append(back * s["residual_scale"])
        sums["dw_post"] = sums.get("dw_post", 0) + (back * k * a).sum(0)
        if gate is not None:
            dgate.index_add_(0, group, back * a * w_post)
        q = back * k * w_post
        whole["du"].append((q - a * (q * a).sum(1, keepdim=True) / D) / size)
    out = {k: torch.cat(v) for k, v in whole.items() if v}
    if dgate is not None and "dy" in s:
        out["dgate"] = dgate
    return {**out, **sums}


def _exact_adamw(s):
    t = s["steps"] + 1
    g = torch.zeros(s["params"].numel(), dtype=torch.float64, device="cuda")
    for i, n, x in zip(s["starts"], s["sizes"], s["grads"]):
        g[i:i + n] = x.reshape(-1).double() * s["grad_scale"].double()
    m, v = s["exp_avg"].double(), s["exp_avg_sq"].double()
    if s["bits"] == 8:
        m = m * s["exp_avg_scale"].double().repeat_interleave(_BLOCK)
        v = (v * s["exp_avg_sq_scale"].double().repeat_interleave(_BLOCK)).square()
    m = torch.lerp(g, m, _BETAS[0])
    v = torch.lerp(g.square(), v, _BETAS[1])
    p = s["params"].double()
    p = p - s["lr"] * (_DECAY * p + m / (1 - _BETAS[0] ** t) / ((v / (1 - _BETAS[1] ** t)).sqrt() + _EPS))
    out = {"params": p}
    if s["bits"] == 32:
        out.update(exp_avg=m, exp_avg_sq=v)
    else:      # rounded at random: the stored codes have no value of their own in 64 bits
        out.update(exp_avg=None, exp_avg_sq=None, exp_avg_scale=None, exp_avg_sq_scale=None)
    if "copies" in s:
        out["copies"] = p
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "norm": _exact_norm, "adamw": _exact_adamw}[case["op"]](s)
