"""What stands between a language model's linear layers and behind its token log probabilities, and the calls their speed is judged by.

  attention   sdgp_attention (+ _bwd): softmax attention of packed sequences, grouped heads, causal or not; prompts, training
              batches and single tokens against a cache
  rotary      sdgp_rotary: queries and keys turned by their positions on one or several axes, and their gradients turned back
  policy      sdgp_policy_loss (+ _bwd): the clipped policy loss with a KL term, from the log probabilities of sdgp_token_logprobs
  preference  sdgp_preference_loss (+ _bwd): the loss of preferred against rejected sequences, from the same log probabilities

``run`` computes each either in plain torch, 32 bits throughout (64 for angles, long sums and what lies next to a border) and
rounded once at the end (``own`` false), or with this library's kernels (``own`` true).  ``exact`` is the definition in 64 bits.
"""
import math
import random

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_CLIP = (0.2, 0.28)


# ------------------------------------------------------------------------------------------------------------- cases

def _attention(name, mode, dtype, heads, kv_heads, D, seqs, lo, hi, shape_seed, causal=True, ahead=0):
    """mode train and prompt: `seqs` sequences of lo .. hi tokens (`ahead` keys in front of each one's queries at most);
    decode: one token of each against a cache of hi places with lo .. hi filled."""
    c = {"op": "attention", "mode": mode, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "D": D, "seqs": seqs, "lo": lo, "hi": hi,
         "shape_seed": shape_seed, "causal": causal, "ahead": ahead}
    return dict(c, name=name) if name else c


def _rotary(name, tokens, dtype, heads, kv_heads, D, axes, interleaved, first, train):
    c = {"op": "rotary", "tokens": tokens, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "D": D, "axes": ",".join(map(str, axes)),
         "interleaved": interleaved, "first": first, "train": train}
    return dict(c, name=name) if name else c


def _policy(name, seqs, lo, hi, shape_seed, average, each, ref=True, masked=0.1):
    c = {"op": "policy", "seqs": seqs, "lo": lo, "hi": hi, "shape_seed": shape_seed, "average": average, "each": each, "ref": ref,
         "masked": masked}
    return dict(c, name=name) if name else c


def _preference(name, seqs, lo, hi, shape_seed, average, smoothing, ref=True, masked=0.3):
    c = {"op": "preference", "seqs": seqs, "lo": lo, "hi": hi, "shape_seed": shape_seed, "average": average, "smoothing": smoothing,
         "ref": ref, "masked": masked}
    return dict(c, name=name) if name else c


def listed():
    return [
        # training on the repository's small token model: 64 sequences of 32 tokens, four heads of its width
        _attention("attn_train_64x32", "train", "bf16", 4, 4, 64, 64, 32, 32, 1),
        # fp32, odd lengths, an odd head size, three queries to a key head
        _attention("attn_train_f32_5_odd", "train", "f32", 6, 2, 80, 5, 101, 1001, 2),
        # pre-training on documents of different lengths packed into one row of 22294 tokens
        _attention("attn_train_packed_22294", "train", "bf16", 16, 4, 128, 8, 100, 4096, 5),
        # serving: a long prompt in one piece
        _attention("attn_prompt_16384", "prompt", "bf16", 32, 8, 128, 1, 16384, 16384, 4),
        # serving: the next token of 32 sequences whose caches are filled unevenly
        _attention("attn_decode_32x8192", "decode", "bf16", 32, 8, 128, 32, 200, 8192, 5),
        # serving: one token each of 16 sequences, far into their contexts
        _rotary("rotary_decode_16", 16, "bf16", 32, 8, 128, (64,), False, 120000, False),
        # video: 9001 patches at (time, height, width), pairs side by side, fp32, and the gradients
        _rotary("rotary_video_f32_9001", 9001, "f32", 12, 12, 80, (8, 16, 16), True, 0, True),
        # pre-training: the queries and keys of a batch of 32768 tokens, and their gradients
        _rotary("rotary_train_32768", 32768, "bf16", 32, 8, 128, (64,), False, 0, True),
        # a small policy step: 64 answers of up to 200 tokens, one advantage each
        _policy("policy_64x200", 64, 20, 200, 6, "sequences", "sequence"),
        # long answers, advantages for each token, averaged over all tokens
        _policy("policy_512x8192", 512, 6000, 9000, 7, "tokens", "token"),
        # a small step over 16 pairs of answers
        _preference("preference_32x300", 32, 50, 300, 8, False, 0.0),
        # 256 pairs of long answers, length-normalised, labels smoothed
        _preference("preference_512x4000", 512, 500, 4000, 9, True, 0.1),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "rotary", "policy", "preference"])
    shape_seed = rng.randrange(1 << 30)
    if op == "attention":
        D = rng.choice([64, 64, 128, 128, 128, 32, 80, 96, 40])
        kv_heads = rng.choice([1, 2, 4, 8])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
        mode = rng.choice(["train", "train", "prompt", "decode"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if mode == "decode":
            hi = _spread(rng, 16, 16384)
            seqs = _spread(rng, 1, max(1, min(128, (1 << 18) // hi)))
            return _attention(None, mode, dtype, heads, kv_heads, D, seqs, rng.choice([0, 1, hi // 4, hi]), hi, shape_seed)
        hi = _spread(rng, 1, 4096 if dtype == "bf16" else 1500)
        seqs = _spread(rng, 1, max(1, min(64, (1 << 24) // (hi * hi), (1 << 14) // hi)))
        return _attention(None, mode, dtype, heads, kv_heads, D, seqs, rng.choice([1, max(1, hi // 3), hi]), hi, shape_seed,
                          rng.random() < 0.75, rng.choice([0, 0, 0, 17, 300]))
    if op == "rotary":
        D = 2 * _spread(rng, 4, 128)
        pairs = rng.choice([D // 2, D // 2, max(1, D // 4)])
        axes = (pairs,)
        if pairs >= 3 and rng.random() < 0.5:
            a = rng.randint(1, pairs - 2)
            b = rng.randint(1, pairs - a - 1)
            axes = (a, b, pairs - a - b)
        kv_heads = rng.choice([1, 2, 4, 8, 0])
        heads = max(1, kv_heads) * rng.choice([1, 3, 4, 8])
        tokens = _spread(rng, 1, max(1, min(32768, (1 << 27) // ((heads + kv_heads) * D))))
        return _rotary(None, tokens, rng.choice(["f32", "bf16"]), heads, kv_heads, D, axes, rng.random() < 0.5, rng.choice([0, 0, 5000, 1000000]),
                       rng.random() < 0.6)
    hi = _spread(rng, 1, 16384)
    seqs = 2 * _spread(rng, 1, max(1, min(256, (1 << 20) // hi)))
    lo = rng.choice([1, max(1, hi // 4), hi])
    masked = rng.choice([0.0, 0.1, 0.6])
    if op == "policy":
        return _policy(None, seqs, lo, hi, shape_seed, rng.choice(["tokens", "sequences"]), rng.choice(["token", "sequence"]),
                       rng.random() < 0.7, masked)
    return _preference(None, seqs, lo, hi, shape_seed, rng.random() < 0.5, rng.choice([0.0, 0.1]), rng.random() < 0.7, masked)


# ------------------------------------------------------------------------------------------------------------ inputs

def _lens(case):
    rng = random.Random(case["shape_seed"])
    return [rng.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]


def _attention_lens(case):
    """(query lengths, key lengths)"""
    lens = _lens(case)
    if case["mode"] == "decode":
        return [1] * len(lens), lens
    rng = random.Random(case["shape_seed"] + 1)
    return lens, [n + rng.randint(0, case["ahead"]) for n in lens]


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 29)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _rand(g, *shape):
    return torch.rand(*shape, device="cuda", generator=g)


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _prepare_attention(case, g):
    dt, H, Hk, D = _DT[case["dtype"]], case["heads"], case["kv_heads"], case["D"]
    lens_q, lens_k = _attention_lens(case)
    state = {"causal": case["causal"], "scale": D ** -0.5, "lens_q": lens_q, "lens_k": lens_k, "offsets": None, "offsets_k": None,
             "lengths": None}
    if case["mode"] == "decode":                  # a cache of equal places, of which each sequence has filled its part
        B, L = case["seqs"], case["hi"]
        state["q"] = (_randn(g, B, 1, H, D) * 1.5).to(dt)
        state["k"], state["v"] = (_randn(g, B, L, Hk, D).to(dt) for _ in range(2))
        state["lengths"] = torch.tensor(lens_k, dtype=torch.int32, device="cuda")
        return state
    Tq, Tk = sum(lens_q), sum(lens_k)
    state["offsets"] = _offsets(lens_q)
    if lens_q == lens_k:                          # cut out of one product's output, as a layer leaves them
        qkv = _randn(g, Tq, H + 2 * Hk, D)
        qkv[:, :H] *= 1.5
        state["q"], state["k"], state["v"] = qkv.to(dt).split((H, Hk, Hk), 1)
    else:
        state["offsets_k"] = _offsets(lens_k)
        state["q"] = (_randn(g, Tq, H, D) * 1.5).to(dt)
        state["k"], state["v"] = _randn(g, Tk, 2 * Hk, D).to(dt).split((Hk, Hk), 1)
    if case["mode"] == "train":
        state["do"] = (_randn(g, Tq, H, D) * 1e-3).to(dt)
    return state


def _prepare_rotary(case, g):
    dt, H, Hk, D, T = _DT[case["dtype"]], case["heads"], case["kv_heads"], case["D"], case["tokens"]
    axes = tuple(map(int, case["axes"].split(",")))
    qkv = _randn(g, T, H + 2 * Hk, D).to(dt)
    state = {"q": qkv[:, :H], "k": qkv[:, H:H + Hk] if Hk else None, "axes": axes, "interleaved": case["interleaved"]}
    # each axis from one radian a place down to 1/10000 of it
    state["freqs"] = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in axes]).float().cuda()
    if len(axes) == 1:
        state["positions"] = case["first"] + torch.arange(T, device="cuda") if T > 64 else torch.randint(0, case["first"] + T, (T,), device="cuda", generator=g)
    else:
        side = max(1, round(T ** (1 / len(axes))))
        at = torch.arange(T, device="cuda")
        state["positions"] = torch.stack([case["first"] + at // side ** (len(axes) - 1)] +
                                         [at // side ** i % side for i in reversed(range(len(axes) - 1))], 1)
    if case["train"]:
        state["dq"] = (_randn(g, T, H, D) * 1e-3).to(dt)
        state["dk"] = (_randn(g, T, Hk, D) * 1e-3).to(dt) if Hk else None
    return state


def _prepare_sequences(case, g):
    """Log probabilities of tokens as a model gives them, those of the policy that sampled them a few updates ago and of the
    reference, prompt tokens masked (their values are not numbers anyone computed)."""
    lens = _lens(case)
    T = sum(lens)
    state = {"offsets": _offsets(lens), "logp": -torch.exp(_randn(g, T) - 1)}
    state["mask"] = _rand(g, T) >= case["masked"] if case["masked"] else None
    state["ref"] = state["logp"] + 0.15 * _randn(g, T) if case["ref"] else None
    if case["op"] == "policy":
        state["old"] = state["logp"] + 0.12 * _randn(g, T)
        state["advantages"] = _randn(g, T if case["each"] == "token" else len(lens))
        state["kl"] = 0.04 if case["ref"] else 0.0
    else:
        state["beta"], state["smoothing"] = (2.0 if case["average"] else 0.1), case["smoothing"]
        state["margin"] = 0.0 if case["ref"] else 0.5
    state["average"] = case["average"]
    if state["mask"] is not None:
        for key in ("old", "ref"):
            if state.get(key) is not None:
                state[key] = torch.where(state["mask"], state[key], math.nan)
    state["g"] = 0.5 + _rand(g, 1)[0]
    return state


_PREPARE = {"attention": _prepare_attention, "rotary": _prepare_rotary, "policy": _prepare_sequences, "preference": _prepare_sequences}


def prepare(case, seed):
    return {"op": case["op"], **_PREPARE[case["op"]](case, _generator(seed))}


# ------------------------------------------------------------------------------------------------------- plain forms

def _groups(lens_q, lens_k, heads):
    """Consecutive sequences, padded to the longest of them, as many as keep the scores below 2^31 values."""
    first, most_q, most_k = 0, 0, 0
    for i, (a, b) in enumerate(zip(lens_q, lens_k)):
        q, k = max(most_q, a), max(most_k, b)
        if i > first and (i + 1 - first) * heads * q * k > 1 << 31:
            yield first, i
            first, q, k = i, a, b
        most_q, most_k = q, k
    yield first, len(lens_q)


def _padded(x, offsets, first, end, most):
    """Rows of sequences first .. end - 1 side by side, [n, most, ...] in fp32, and where they are in x (the last row for none)."""
    at = offsets[first:end, None] + torch.arange(most, device=x.device)
    there = at < offsets[first + 1:end + 1, None]
    return torch.where(there[..., None, None], x[at.clamp(max=x.shape[0] - 1)].float(), 0.0), at, there


def _attend(q, k, v, there, causal, scale, lens_q, lens_k, do):
    """q [n, Lq, H, D], k and v [n, Lk, Hk, D] in fp32, there [n, Lk]: which keys there are."""
    n, Lq, H, D = q.shape
    Lk, Hk = k.shape[1], k.shape[2]
    G = H // Hk
    rows = lambda x: x.view(n, Lq, Hk, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hk, G * Lq, D)  # noqa: E731
    back = lambda x: x.view(n, Hk, G, Lq, D).permute(0, 3, 1, 2, 4).reshape(n, Lq, H, D)  # noqa: E731
    qh, kh, vh = rows(q), k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
    seen = there[:, None, :]
    if causal:                                            # the last query sees the last key
        i = torch.arange(Lq, device=q.device)[None, :, None] + (lens_k - lens_q)[:, None, None]
        seen = seen & (torch.arange(Lk, device=q.device) <= i)
    seen = seen[:, None, None].expand(n, 1, G, Lq if causal else 1, Lk).expand(n, 1, G, Lq, Lk).reshape(n, 1, G * Lq, Lk)
    s = (qh @ kh.transpose(2, 3)) * scale
    s.masked_fill_(~seen, -math.inf)
    top = s.amax(3, keepdim=True) if Lk else s.new_full((n, Hk, G * Lq, 1), -math.inf)
    p = s.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(3, keepdim=True)
    p /= torch.where(total > 0, total, 1.0)
    o = p @ vh
    lse = (top + torch.log(total)).view(n, Hk, G, Lq).permute(0, 3, 1, 2).reshape(n, Lq, H)
    if do is None:
        return back(o), lse
    dh = rows(do)
    dv = p.transpose(2, 3) @ dh
    ds = p * (dh @ vh.transpose(2, 3) - (dh * o).sum(3, keepdim=True))
    dq = (ds @ kh) * scale
    dk = (ds.transpose(2, 3) @ qh) * scale
    return back(o), lse, back(dq), dk.transpose(1, 2), dv.transpose(1, 2)


def _plain_attention(s):
    q, k, v = s["q"], s["k"], s["v"]
    dt = q.dtype
    if s["lengths"] is not None:
        there = torch.arange(k.shape[1], device=k.device) < s["lengths"][:, None]
        one = torch.ones_like(s["lengths"])
        v = torch.where(there[..., None, None], v.float(), 0.0)
        o, lse = _attend(q.float(), k.float(), v, there, s["causal"], s["scale"], one, s["lengths"], None)
        return {"o": o.to(dt), "lse": lse}
    off_q, off_k = s["offsets"], s["offsets_k"] if s["offsets_k"] is not None else s["offsets"]
    lens_q, lens_k = off_q.diff(), off_k.diff()
    train = "do" in s
    out = {"o": torch.empty(q.shape, dtype=dt, device=q.device), "lse": torch.empty(q.shape[:2], device=q.device)}
    if train:
        out.update(dq=torch.empty(q.shape, dtype=dt, device=q.device), dk=torch.empty(k.shape, dtype=dt, device=q.device),
                   dv=torch.empty(k.shape, dtype=dt, device=q.device))
    for first, end in _groups(s["lens_q"], s["lens_k"], q.shape[1]):
        Lq, Lk = max(s["lens_q"][first:end]), max(s["lens_k"][first:end])
        qp, at_q, in_q = _padded(q, off_q, first, end, Lq)
        kp, at_k, in_k = _padded(k, off_k, first, end, Lk)
        vp = _padded(v, off_k, first, end, Lk)[0]
        do = _padded(s["do"], off_q, first, end, Lq)[0] if train else None
        # as many key heads at a time as keep the scores below 2^31 values
        per, Hk = q.shape[1] // k.shape[1], k.shape[1]
        step = max(1, min(Hk, (1 << 31) // max(1, (end - first) * per * Lq * Lk)))
        parts = [_attend(qp[:, :, h * per:(h + step) * per], kp[:, :, h:h + step], vp[:, :, h:h + step], in_k, s["causal"], s["scale"],
                         lens_q[first:end], lens_k[first:end], None if do is None else do[:, :, h * per:(h + step) * per])
                 for h in range(0, Hk, step)]
        for key, *got in zip(out, *parts):
            x = torch.cat(got, 2)
            at, there = (at_k, in_k) if key in ("dk", "dv") else (at_q, in_q)
            out[key][at[there]] = x[there].to(out[key].dtype)
    return out


def _turn(x, cos, sin, interleaved):
    """The first 2 F values of every head turned; cos, sin [T, F]."""
    F = cos.shape[1]
    y = x.float().clone()
    a, b = (y[..., 0:2 * F:2], y[..., 1:2 * F:2]) if interleaved else (y[..., :F], y[..., F:2 * F])
    c, s = cos[:, None], sin[:, None]
    first, second = a * c - b * s, a * s + b * c
    a.copy_(first)
    b.copy_(second)
    return y.to(x.dtype)


def _plain_rotary(s):
    axis = torch.cat([torch.full((n,), i, device="cuda") for i, n in enumerate(s["axes"])])
    at = s["positions"] if s["positions"].dim() == 2 else s["positions"][:, None]
    angle = at[:, axis].double() * s["freqs"].double()                   # far positions: many turns
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = {"q": _turn(s["q"], cos, sin, s["interleaved"])}
    if s["k"] is not None:
        out["k"] = _turn(s["k"], cos, sin, s["interleaved"])
    if "dq" in s:
        out["dq"] = _turn(s["dq"], cos, -sin, s["interleaved"])
        if s["k"] is not None:
            out["dk"] = _turn(s["dk"], cos, -sin, s["interleaved"])
    return out


def _sums(x, offsets):
    """Sums over the sequences, in 64 bits."""
    c = torch.cat([x.new_zeros(1, dtype=torch.float64), x.double().cumsum(0)])
    return c[offsets[1:].long()] - c[offsets[:-1].long()]


def _sequence_of(offsets, T):
    return torch.bucketize(torch.arange(T, device=offsets.device), offsets[1:].long(), right=True)


def _plain_policy(s):
    logp, old, offsets = s["logp"], s["old"], s["offsets"]
    T = logp.numel()
    seq = _sequence_of(offsets, T)
    on = s["mask"] if s["mask"] is not None else torch.ones(T, dtype=torch.bool, device="cuda")
    A = s["advantages"] if s["advantages"].numel() == T else s["advantages"][seq]
    d = torch.where(on, logp.double() - old.double(), 0.0)               # which side of the border: in 64 bits
    lo, hi = math.log1p(-_CLIP[0]), math.log1p(_CLIP[1])
    cut = on & (((A > 0) & (d > hi)) | ((A < 0) & (d < lo)))
    r = torch.exp(d.float())
    loss = -A * torch.where(cut, torch.where(A > 0, 1 + _CLIP[1], 1 - _CLIP[0]), r)
    grad = torch.where(cut, 0.0, -A * r)
    kl = torch.zeros_like(logp)
    if s["ref"] is not None:
        x = torch.where(on, s["ref"].double() - logp.double(), 0.0)
        kl = (torch.expm1(x) - x).float()                                # small differences: e^x - 1 - x cancels
        loss = loss + s["kl"] * kl
        grad = grad - s["kl"] * torch.expm1(x).float()
    zero = torch.zeros_like(loss)
    count, lsum, ksum, csum = (_sums(torch.where(on, x, zero), offsets) for x in (torch.ones_like(loss), loss, kl, cut.float()))
    total = count.sum()
    if s["average"] == "tokens":
        each = torch.ones_like(count) / total.clamp(min=1)
    else:
        each = torch.where(count > 0, 1 / count.clamp(min=1), 0.0) / (count > 0).sum().clamp(min=1)
    share = 1 / total.clamp(min=1)
    dlogp = torch.where(on, grad * (each.float() * s["g"])[seq], zero)
    return {"loss": (lsum * each).sum().float(), "kl": (ksum.sum() * share).float(), "clipped": (csum.sum() * share).float(), "dlogp": dlogp}


def _plain_preference(s):
    logp, offsets = s["logp"], s["offsets"]
    T = logp.numel()
    on = s["mask"] if s["mask"] is not None else torch.ones(T, dtype=torch.bool, device="cuda")
    x = logp.double() if s["ref"] is None else logp.double() - s["ref"].double()
    sums = _sums(torch.where(on, x, 0.0), offsets)
    each = torch.ones_like(sums)
    if s["average"]:
        each = 1 / _sums(on.float(), offsets).clamp(min=1)
    score = s["beta"] * sums * each
    z = score[0::2] - score[1::2] - s["margin"]
    eps = s["smoothing"]
    soft = lambda a: torch.log1p(torch.exp(-a.abs())) + (-a).clamp(min=0)  # noqa: E731   -ln sigmoid(a)
    pairs = z.numel()
    loss = ((1 - eps) * soft(z) + eps * soft(-z)).sum() / pairs
    dz = (eps - 1 / (1 + torch.exp(z))) / pairs                          # = eps sigmoid(z) - (1 - eps) sigmoid(-z), over the pairs
    w = torch.stack([dz, -dz], 1).view(-1) * s["beta"] * each
    dlogp = torch.where(on, (w.float() * s["g"])[_sequence_of(offsets, T)], 0.0)
    return {"loss": loss.float(), "margins": z.float(), "dlogp": dlogp}


# ---------------------------------------------------------------------------------------------- the library's kernels

def _own_attention(s):
    import paper_2202_00774_amd as sdgp
    at = (s["offsets"], s["offsets_k"])
    o, lse = sdgp.sdgp_attention(s["q"], s["k"], s["v"], *at, lengths=s["lengths"], causal=s["causal"], scale=s["scale"])
    out = {"o": o, "lse": lse}
    if "do" in s:
        out["dq"], out["dk"], out["dv"] = sdgp.sdgp_attention_bwd(s["do"], s["q"], s["k"], s["v"], o, lse, *at, causal=s["causal"],
                                                                  scale=s["scale"])
    return out


def _own_rotary(s):
    import paper_2202_00774_amd as sdgp
    how = (s["positions"], s["freqs"], s["axes"])
    q, k = sdgp.sdgp_rotary(s["q"], s["k"], *how, interleaved=s["interleaved"])
    out = {"q": q} if k is None else {"q": q, "k": k}
    if "dq" in s:
        dq, dk = sdgp.sdgp_rotary(s["dq"], s["dk"], *how, interleaved=s["interleaved"], inverse=True)
        out.update({"dq": dq} if dk is None else {"dq": dq, "dk": dk})
    return out


def _own_policy(s):
    import paper_2202_00774_amd as sdgp
    given = (s["logp"], s["old"], s["advantages"], s["ref"], s["mask"], s["offsets"])
    how = {"clip": _CLIP, "kl": s["kl"], "average": s["average"]}
    loss, kl, clipped, weights = sdgp.sdgp_policy_loss(*given, **how)
    return {"loss": loss, "kl": kl, "clipped": clipped, "dlogp": sdgp.sdgp_policy_loss_bwd(s["g"], weights, *given, **how)}


def _own_preference(s):
    import paper_2202_00774_amd as sdgp
    loss, margins, weights = sdgp.sdgp_preference_loss(s["logp"], s["ref"], s["mask"], s["offsets"], beta=s["beta"], margin=s["margin"],
                                                       smoothing=s["smoothing"], average=s["average"])
    return {"loss": loss, "margins": margins, "dlogp": sdgp.sdgp_preference_loss_bwd(s["g"], weights, s["logp"], s["mask"], s["offsets"])}


def run(state):
    if own:
        return {"attention": _own_attention, "rotary": _own_rotary, "policy": _own_policy, "preference": _own_preference}[state["op"]](state)
    return {"attention": _plain_attention, "rotary": _plain_rotary, "policy": _plain_policy, "preference": _plain_preference}[state["op"]](state)


# -------------------------------------------------------------------------------------------------------------- work

def work(case):
    if case["op"] == "attention":
        H, Hk, D, size, train = case["heads"], case["kv_heads"], case["D"], _SIZE[case["dtype"]], case["mode"] == "train"
        lens_q, lens_k = _attention_lens(case)
        pairs = 0
        for a, b in zip(lens_q, lens_k):
            if case["causal"]:                       # the queries behind the first a - b see 1, 2, .. or b - a + 1, .. keys
                n = min(a, b)
                pairs += n * (b - n) + n * (n + 1) // 2
            else:
                pairs += a * b
        Tq, Tk = sum(lens_q), sum(lens_k)
        values = Tq * H * D * (4 if train else 2) + Tk * Hk * D * (4 if train else 2)   # q o do dq | k v dk dv
        return {"bytes": values * size + Tq * H * 4, "flops": pairs * H * D * (14 if train else 4)}
    if case["op"] == "rotary":
        axes = tuple(map(int, case["axes"].split(",")))
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        times = 2 if case["train"] else 1
        return {"bytes": times * 2 * n * case["D"] * _SIZE[case["dtype"]] + case["tokens"] * 8 * len(axes),
                "flops": times * n * 6 * sum(axes)}
    lens = _lens(case)
    T, S = sum(lens), len(lens)
    tokens = 1 + (1 if case["ref"] else 0) + (0.25 if case["masked"] else 0) + 1           # logp, ref, mask | dlogp
    if case["op"] == "policy":
        tokens += 1 + (1 if case["each"] == "token" else 0)
        return {"bytes": int(T * 4 * tokens) + 8 * S, "flops": T * 30}
    return {"bytes": int(T * 4 * tokens) + 12 * S, "flops": T * 5}


# ------------------------------------------------------------------------------------------------------------- exact

def _exact_attention(s):
    """One sequence and one query head at a time, only the queries that see a key; the gradients by torch's own differentiation."""
    decode, train = s["lengths"] is not None, "do" in s
    H, Hk = s["q"].shape[-2], s["k"].shape[-2]
    out = {"o": torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"),
           "lse": torch.full(s["q"].shape[:-1], -math.inf, dtype=torch.float64, device="cuda")}
    if train:
        out.update({"d" + n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"})
    at_q = at_k = 0
    for b, (nq, nk) in enumerate(zip(s["lens_q"], s["lens_k"])):
        blind = (max(0, nq - nk) if s["causal"] else 0) if nk else nq
        rows, keys = ((b, slice(blind, nq)), (b, slice(0, nk))) if decode else ((slice(at_q + blind, at_q + nq),), (slice(at_k, at_k + nk),))
        at_q, at_k = at_q + nq, at_k + nk
        if blind == nq:
            continue
        hidden = torch.ones(nq, nk, dtype=torch.bool, device="cuda").triu(nk - nq + 1)[blind:] if s["causal"] else None
        for h in range(H):
            j = h // (H // Hk)
            q, k, v = (t.double().requires_grad_(train) for t in (s["q"][(*rows, h)], s["k"][(*keys, j)], s["v"][(*keys, j)]))
            z = torch.mm(q, k.t()) * s["scale"]
            if hidden is not None:
                z = z.masked_fill(hidden, -math.inf)
            o = torch.mm(torch.softmax(z, 1), v)
            out["o"][(*rows, h)] = o.detach()
            out["lse"][(*rows, h)] = torch.logsumexp(z.detach(), 1)
            if train:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), s["do"][(*rows, h)].double())
                out["dq"][(*rows, h)] = dq
                out["dk"][(*keys, j)] += dk
                out["dv"][(*keys, j)] += dv
    return out


def _exact_rotary(s):
    """Pairs as complex numbers times e^(i angle)."""
    F = s["freqs"].numel()
    at = s["positions"].view(s["positions"].shape[0], -1).double()
    per_axis = torch.split(s["freqs"].double(), s["axes"])
    angle = torch.cat([at[:, i:i + 1] * f for i, f in enumerate(per_axis)], 1)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]

    def turned(x, unit):
        x = x.double()
        head, rest = x[..., :2 * F], x[..., 2 * F:]
        pairs = head.unflatten(-1, (F, 2)) if s["interleaved"] else head.unflatten(-1, (2, F)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
        head = z.flatten(-2) if s["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([head, rest], -1)

    out = {}
    for key, u in (("q", unit), ("k", unit), ("dq", unit.conj()), ("dk", unit.conj())):
        if s.get(key) is not None:
            out[key] = turned(s[key], u)
    return out


def _exact_policy(s):
    """The gradient by torch's own differentiation; the sequences one by one."""
    ends = s["offsets"].tolist()
    T = ends[-1]
    logp = s["logp"].double().requires_grad_()
    A = s["advantages"].double()
    lens = torch.tensor([b - a for a, b in zip(ends, ends[1:])], device="cuda")
    A = A if A.numel() == T else torch.repeat_interleave(A, lens)
    on = s["mask"] if s["mask"] is not None else torch.ones(T, dtype=torch.bool, device="cuda")
    ratio = torch.exp(logp[on] - s["old"].double()[on])
    a = A[on]
    kept = torch.minimum(ratio * a, ratio.clamp(1 - _CLIP[0], 1 + _CLIP[1]) * a)
    kl = torch.zeros_like(kept)
    if s["ref"] is not None:
        x = s["ref"].double()[on] - logp[on]
        kl = torch.expm1(x) - x
    each = s["kl"] * kl - kept
    if s["average"] == "tokens":
        loss = each.mean() if each.numel() else each.sum()
    else:
        means = [part.mean() for part in each.split([int(on[i:j].sum()) for i, j in zip(ends, ends[1:])]) if part.numel()]
        loss = torch.stack(means).mean() if means else each.sum()
    grad = torch.autograd.grad(loss, logp)[0] * s["g"].double()
    # the share whose ratio is cut: which side of a border is decided by the ratio itself
    outside = torch.where(a > 0, ratio > 1 + _CLIP[1], (a < 0) & (ratio < 1 - _CLIP[0]))
    n = max(1, each.numel())
    return {"loss": loss.detach(), "kl": kl.detach().sum() / n, "clipped": outside.double().sum() / n, "dlogp": grad}


def _exact_preference(s):
    ends = s["offsets"].tolist()
    logp = s["logp"].double().requires_grad_()
    x = logp if s["ref"] is None else logp - s["ref"].double()
    scores = []
    for i, j in zip(ends, ends[1:]):
        part = x[i:j] if s["mask"] is None else x[i:j][s["mask"][i:j]]
        scores.append(part.mean() if s["average"] and part.numel() else part.sum())
    scores = s["beta"] * torch.stack(scores)
    z = scores.view(-1, 2)[:, 0] - scores.view(-1, 2)[:, 1] - s["margin"]
    eps = s["smoothing"]
    loss = -((1 - eps) * torch.nn.functional.logsigmoid(z) + eps * torch.nn.functional.logsigmoid(-z)).mean()
    grad = torch.autograd.grad(loss, logp)[0] * s["g"].double()
    return {"loss": loss.detach(), "margins": z.detach(), "dlogp": grad}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "rotary": _exact_rotary, "policy": _exact_policy, "preference": _exact_preference}[case["op"]](s)
