"""Plain 64-bit forms of the sequence-layer operators and bounds on their rounding, for the
operators' tests (torch float64 on the CPU; every sum written out from its definition).

The bounds count roundings of half a step, u = eps / 2 of a type (bf16 2^-8, fp16 2^-11,
fp32 2^-24), against sums of magnitudes: a sum of n fp32 products is off by at most
(n + 2) 2^-24 of the sum of their magnitudes.
"""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def _pairs(q, k, v, g, scale):
    """One sequence and head in its own order: decays between rows [L, L] (lower part) and the
    running sums of the log decays."""
    b = torch.cumsum(g, 0)
    low = torch.ones(len(g), len(g), dtype=torch.bool).tril()
    d = torch.where(low, torch.exp(torch.where(low, b[:, None] - b[None, :], torch.zeros(()).double())), torch.zeros(()).double())
    return d, b


def attention(q, k, v, g, offsets, scale, reverse=False, s0=None, d_out=None, d_state=None):
    """Values and magnitudes of decay_attention, and of its backward pass if d_out is given.

    q, k [R, Hk, dk], v [R, H, dv], g [R, H] or [H], all float64.  Returns a dict name ->
    (value, magnitude, weight magnitude): the magnitude has every product's absolute value, the
    weight magnitude the absolute values of the weights (of pairs of rows) times the vectors'."""
    rows, hk, dk = q.shape
    h, dv = v.shape[1], v.shape[2]
    n = len(offsets) - 1
    group = h // hk
    gg = g.expand(rows, h) if g.dim() == 1 else g
    names = ["out", "state"] if d_out is None else ["dq", "dk", "dv", "dg", "d_initial"]
    shape = {"out": (rows, h, dv), "state": (n, h, dk, dv), "dq": (rows, hk, dk), "dk": (rows, hk, dk),
             "dv": (rows, h, dv), "dg": (rows, h), "d_initial": (n, h, dk, dv)}
    r = {x: [torch.zeros(shape[x]).double() for _ in range(3)] for x in names}
    for i in range(n):
        at = torch.arange(offsets[i], offsets[i + 1])
        if reverse:
            at = at.flip(0)
        for j in range(h):
            Q, K, V, G = q[at, j // group], k[at, j // group], v[at, j], gg[at, j]
            zero = torch.zeros(dk, dv).double()
            S0 = s0[i, j] if s0 is not None else zero
            L = len(at)
            if L == 0:
                if d_out is None:
                    r["state"][0][i, j] = S0
                else:
                    r["d_initial"][0][i, j] = d_state[i, j] if d_state is not None else zero
                continue
            d, b = _pairs(Q, K, V, G, scale)
            eb = torch.exp(b)[:, None]                      # from before the first row to each row
            ee = torch.exp(b[-1] - b)[:, None]              # from each row to the last
            A, aA = (Q @ K.T) * d, (Q.abs() @ K.abs().T) * d
            if d_out is None:
                r["out"][0][at, j] = scale * (A @ V + eb * (Q @ S0))
                r["out"][1][at, j] = abs(scale) * (aA @ V.abs() + eb * (Q.abs() @ S0.abs()))
                r["out"][2][at, j] = abs(scale) * (A.abs() @ V.abs())
                r["state"][0][i, j] = torch.exp(b[-1]) * S0 + K.T @ (ee * V)
                r["state"][1][i, j] = torch.exp(b[-1]) * S0.abs() + K.abs().T @ (ee * V.abs())
                continue
            D = d_out[at, j]
            T = d_state[i, j] if d_state is not None else zero
            B, aB = (D @ V.T) * d, (D.abs() @ V.abs().T) * d
            hh = j // group
            r["dq"][0][at, hh] += scale * (B @ K + eb * (D @ S0.T))
            r["dq"][1][at, hh] += abs(scale) * (aB @ K.abs() + eb * (D.abs() @ S0.abs().T))
            r["dq"][2][at, hh] += abs(scale) * (B.abs() @ K.abs())
            r["dk"][0][at, hh] += scale * (B.T @ Q) + ee * (V @ T.T)
            r["dk"][1][at, hh] += abs(scale) * (aB.T @ Q.abs()) + ee * (V.abs() @ T.abs().T)
            r["dk"][2][at, hh] += abs(scale) * (B.T.abs() @ Q.abs())
            r["dv"][0][at, j] = scale * (A.T @ D) + ee * (K @ T)
            r["dv"][1][at, j] = abs(scale) * (aA.T @ D.abs()) + ee * (K.abs() @ T.abs())
            r["dv"][2][at, j] = abs(scale) * (A.T.abs() @ D.abs())
            r["d_initial"][0][i, j] = torch.exp(b[-1]) * T + scale * (Q * eb).T @ D
            r["d_initial"][1][i, j] = torch.exp(b[-1]) * T.abs() + abs(scale) * (Q.abs() * eb).T @ D.abs()
            # g_u is in the decay between rows s < u <= t, in that from before the first row to t >= u, and
            # in that from s < u to the last row
            M = scale * (Q @ K.T) * (D @ V.T) * d
            aM = abs(scale) * (Q.abs() @ K.abs().T) * (D.abs() @ V.abs().T) * d
            first = scale * eb[:, 0] * ((Q @ S0) * D).sum(1)
            afirst = abs(scale) * eb[:, 0] * ((Q.abs() @ S0.abs()) * D.abs()).sum(1)
            last = ee[:, 0] * ((K @ T) * V).sum(1)
            alast = ee[:, 0] * ((K.abs() @ T.abs()) * V.abs()).sum(1)
            both, aboth = torch.exp(b[-1]) * (T * S0).sum(), torch.exp(b[-1]) * (T * S0).abs().sum()
            # the kernel's sums run over rows and cancel within a span: their roundings are of all that is in them
            total = aM.sum() + afirst.sum() + alast.sum() + aboth
            for u in range(L):
                r["dg"][0][at[u], j] = M[u:, :u].sum() + first[u:].sum() + last[:u].sum() + both
                r["dg"][1][at[u], j] = total
    return {x: tuple(y) for x, y in r.items()}


def attention_bound(name, dtype, ref, length):
    """What an output may be off: its own rounding, the rounding of the pairs' weights (bf16), and fp32
    arithmetic: exps of arguments up to ~100 (2^-17 relative), sums over d and the rows, states in two bf16
    parts (2^-16)."""
    value, mag, weights = ref
    u = HALF[dtype]
    if name in ("state", "d_initial", "dg"):
        return (2.0 ** -17 + (length + 256) * 2.0 ** -24) * mag + 1e-30
    t = u * value.abs() + (2.0 ** -16 + (length + 256) * 2.0 ** -24) * mag * (1 + u) + 1e-30
    if dtype == torch.bfloat16:
        t = t + u * (1 + u) * weights
    if dtype == torch.float16:
        t = t + 2.0 ** -25  # half a step of the smallest values
    return t


def norm_rotate(x, gain, pos, rot, base, interleaved, eps, dy=None):
    """x [R, H, d] and positions [R] in 64 bits: the outputs, or (dx, dgain, magnitude of dgain) for dy."""
    d = x.shape[-1]
    j = torch.arange(rot // 2).double()
    a = pos.double()[:, None, None] * base ** (-2 * j / rot)
    c, s = torch.cos(a), torch.sin(a)
    lo = (2 * torch.arange(rot // 2)) if interleaved else torch.arange(rot // 2)
    hi = lo + (1 if interleaved else rot // 2)

    def turn(y, sign):
        z = y.clone()
        z[..., lo] = y[..., lo] * c - sign * y[..., hi] * s
        z[..., hi] = y[..., hi] * c + sign * y[..., lo] * s
        return z

    inv = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if dy is None:
        return turn(x * inv * gain, 1.0)
    dz, xh = turn(dy, -1.0), x * inv
    w = dz * gain
    return inv * (w - xh * (w * xh).mean(-1, keepdim=True)), (dz * xh).sum((0, 1)), (dz * xh).abs().sum((0, 1))


def activation(a, kind):
    if kind == "silu":
        s = torch.sigmoid(a)
        return a * s, s * (1 + a * (1 - s))
    p = 0.5 * torch.erfc(-a / math.sqrt(2.0))
    return a * p, p + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)


def recurrence(q, k, v, g, offsets, scale, reverse=False, s0=None, d_out=None, d_state=None, drop=()):
    """decay_attention and, if d_out is given, its gradients, row by row as the recurrence defines them (float64), for
    sequences of any length.  A row's decay's gradient is e^g <gradient of the state after the row, state before it>.

    q, k [R, Hk, dk], v [R, H, dv], g [R, H].  Returns a dict of "out" (zeros outside of all sequences), "state" and, with
    d_out, "dq", "dk", "dv", "dg", "d_initial".  drop: rows at whose border with the row before the state and its gradient
    are lost, a mistake for the tests to find."""
    rows, hk, dk = q.shape
    h, dv = v.shape[1], v.shape[2]
    n, group = len(offsets) - 1, h // hk
    Q, K = q.repeat_interleave(group, 1), k.repeat_interleave(group, 1)
    r = {"out": torch.zeros_like(v), "state": torch.zeros(n, h, dk, dv).double()}
    if d_out is not None:
        r |= {"dq": torch.zeros_like(Q), "dk": torch.zeros_like(K), "dv": torch.zeros_like(v), "dg": torch.zeros_like(g),
              "d_initial": torch.zeros_like(r["state"])}
    e = torch.exp(g)[:, :, None, None]
    for i in range(n):
        order = list(range(offsets[i], offsets[i + 1]))
        if reverse:
            order.reverse()
        state = torch.zeros(h, dk, dv).double() if s0 is None else s0[i].clone()
        before = []
        for t in order:
            if (t + 1 if reverse else t) in drop:
                state = torch.zeros_like(state)
            if d_out is not None:
                before.append(state)
            state = e[t] * state + K[t][:, :, None] * v[t][:, None, :]
            r["out"][t] = scale * (Q[t][:, None, :] @ state)[:, 0]
            if d_out is not None:
                r["dq"][t] = scale * (state @ d_out[t][:, :, None])[..., 0]
        r["state"][i] = state
        if d_out is None:
            continue
        grad = torch.zeros_like(state) if d_state is None else d_state[i].clone()
        for t, was in zip(reversed(order), reversed(before)):
            grad = grad + scale * Q[t][:, :, None] * d_out[t][:, None, :]
            r["dk"][t] = (grad @ v[t][:, :, None])[..., 0]
            r["dv"][t] = (K[t][:, None, :] @ grad)[:, 0]
            r["dg"][t] = e[t, :, 0, 0] * (grad * was).sum((1, 2))
            grad = e[t] * grad
            if (t + 1 if reverse else t) in drop:
                grad = torch.zeros_like(grad)
        r["d_initial"][i] = grad
    if d_out is not None:
        r["dq"], r["dk"] = (x.view(rows, hk, group, dk).sum(2) for x in (r["dq"], r["dk"]))
    return r


def off(got, want):
    """Two-norm of the difference over the two-norm of what is wanted."""
    return ((got.double().cpu() - want).norm() / want.norm()).item()


# What two-norms may be off.  An output's own rounding, those of the pairs' weights and of the operands are each at most half
# a step, u = HALF[type], and evenly spread over it, so u / sqrt(3) in the two-norm: three of them u.  fp32 sums: at most some
# 250 roundings of 2^-24 in a row (a chunk's products and rows, the steps of a chain), 2^-16 of the magnitudes, which signs at
# random leave a small multiple of in the two-norm.
NORM_FP32 = 2.0 ** -14
NORM = {torch.float32: NORM_FP32, torch.bfloat16: 2.0 ** -8 + NORM_FP32, torch.float16: 2.0 ** -11 + NORM_FP32}
