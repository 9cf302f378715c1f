"""Attention and its gradients in 64 bits, one sequence and query head at a time, with a bound for what the kernels' roundings
can move each value by."""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def attention(q, k, v, spans, causal, scale, do=None):
    """q [Tq, H, D], k and v [Tk, Hk, D]; spans: (first query, end, first key, end) of every sequence.
    Returns {name: (value, bound)}.

    With u half a step of the type (of its products' operands too) and f = 2^-24:
      scores   |ds| <= (D + 8) f max sum |q k| scale, so p is off by E p, E = 2 |ds| + (n + 8) f for n keys (the sum of the
               softmax; exp2 and the logarithm within their few f), and by u p more where it is rounded
      o        sum p |v| (E + u + n f), and u |o| for storing it
      delta    sum |do| (the bound of o) + D f sum |do o|
      dP       D f sum |do v|
      dS       p ((E + u + 2 f) |dP - delta| + the two above)
      dv       sum p |do| (E + u + n f), dq and dk the sums of dS's bounds (and n f |dS|) with |k| and |q|, and u of what is stored"""
    u, f = HALF_STEP[q.dtype], 2.0 ** -24
    operand = 0.0 if q.dtype == torch.float32 else u
    H, D, Hk = q.shape[1], q.shape[2], k.shape[1]
    like = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=t.device)  # noqa: E731
    out = {n: [like(t), like(t)] for n, t in (("o", q), ("lse", q[..., 0]), ("dq", q), ("dk", k), ("dv", k))}
    out["lse"][0].fill_(-math.inf)
    for q0, q1, k0, k1 in spans:
        nq, nk = q1 - q0, k1 - k0
        if not nq or not nk:
            continue
        hidden = torch.ones(nq, nk, dtype=torch.bool, device=q.device).triu(nk - nq + 1) if causal else torch.zeros(nq, nk, dtype=torch.bool, device=q.device)
        for h in range(H):
            j = h // (H // Hk)
            Q, K, V = q[q0:q1, h].double(), k[k0:k1, j].double(), v[k0:k1, j].double()
            s = (Q @ K.T * scale).masked_fill(hidden, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse.clamp(min=-1e300)[:, None])
            off = (D + 8) * f * float((Q.abs() @ K.abs().T * scale).max())
            E = 2 * off + (nk + 8) * f
            A = p @ V.abs()
            o = p @ V
            o_bound = A * (E + operand + nk * f) + u * o.abs()
            out["o"][0][q0:q1, h], out["o"][1][q0:q1, h] = o, o_bound
            out["lse"][0][q0:q1, h], out["lse"][1][q0:q1, h] = lse, off + (nk + 8) * f + 8 * f * lse.abs().clamp(max=1e9)
            if do is None:
                continue
            dO = do[q0:q1, h].double()
            dP, delta = dO @ V.T, (dO * o).sum(1, keepdim=True)
            dS = p * (dP - delta)
            dS_bound = p * ((E + operand + 2 * f) * (dP - delta).abs() + D * f * (dO.abs() @ V.abs().T) +
                            (dO.abs() * (o_bound + D * f * o.abs())).sum(1, keepdim=True))
            n = max(nk, nq * (H // Hk))
            for name, at, head, x, b in (
                    ("dq", slice(q0, q1), h, scale * (dS @ K), scale * ((dS_bound + n * f * dS.abs()) @ K.abs())),
                    ("dk", slice(k0, k1), j, scale * (dS.T @ Q), scale * ((dS_bound + n * f * dS.abs()).T @ Q.abs())),
                    ("dv", slice(k0, k1), j, p.T @ dO, (p * (E + operand + n * f)).T @ dO.abs())):
                out[name][0][at, head] += x
                out[name][1][at, head] += b
    for name in ("dq", "dk", "dv"):
        out[name][1] += u * out[name][0].abs()
    return out


def check(got, out, name):
    value, bound = out[name]
    got = got.double()
    same = torch.isinf(value) & (got == value)
    assert bool(torch.isfinite(torch.where(same, 0.0, got)).all()), f"{name} is not finite everywhere"
    excess = torch.where(same, -1.0, (got - value).abs() - bound)
    worst = int(excess.argmax()) if excess.numel() else 0
    assert not excess.numel() or float(excess.max()) <= 1e-30, \
        f"{name}: off by {float((got - value).abs().flatten()[worst]):.3g}, bound {float(bound.flatten()[worst]):.3g}, value {float(value.flatten()[worst]):.3g} at {worst}"


def spans_of(lens_q, lens_k, first_q=0, first_k=0):
    out = []
    for a, b in zip(lens_q, lens_k):
        out.append((first_q, first_q + a, first_k, first_k + b))
        first_q, first_k = first_q + a, first_k + b
    return out
