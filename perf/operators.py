"""The sequence-layer operators of the track-fit library, as measurable cases.

A layer of a comparison encoder (linear attention with decay over packed hit
sequences, the normalised and rotated queries and keys in front of it, the gated
feed-forward block behind it) is made of three operators.  A case is a dict:

op        "attn"       decay_attention: packed sequences, optional initial and final states
          "attn_bwd"   decay_attention_backward
          "step"       decay_attention_step: one token of every sequence
          "norm"       qk_norm_rotate          "norm_bwd"  qk_norm_rotate_backward
          "ffn"        gated_ffn               "ffn_bwd"   gated_ffn_backward
dtype     "fp32", "bf16" or "fp16": the tensors' type
seqs, len_min, len_max   sequences of the batch; lengths uniform, or (spread) uniform in their logarithm
heads, qk_heads, d_k, d_v   heads of values, decays and outputs; heads of queries and keys; widths
const_decay   one decay a head instead of one a row and head
states    an initial state comes in and the last one goes out (backward: their gradients)
reverse   the recurrence runs from each sequence's last row to its first
rows, q_heads, k_heads, d, rot, interleaved, far   "norm": far positions as of a long stream, else from the rows
rows, width, inner, act   "ffn": rows of x, its width, the block's inner width, the activation
"""
import math

import numpy as np
import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
BASE, EPS = 10000.0, 1e-6


def listed():
    return [
        # one track's next hit, online: the smallest call, latency
        dict(name="step_one_bf16", op="step", dtype="bf16", seqs=1, heads=3, qk_heads=3, d_k=64, d_v=64,
             const_decay=False),
        # the next token of many open sequences, grouped queries and keys
        dict(name="step_512_bf16", op="step", dtype="bf16", seqs=509, heads=16, qk_heads=4, d_k=64, d_v=128,
             const_decay=False),
        # a quarter of a deployment call's tracks through one mixing layer of 192 channels
        dict(name="attn_tracks_bf16", op="attn", dtype="bf16", seqs=65536, len_min=8, len_max=20, spread=False,
             heads=3, qk_heads=3, d_k=64, d_v=64, const_decay=False, states=False, reverse=False),
        # one long sequence, its last state kept for single tokens
        dict(name="attn_long_bf16", op="attn", dtype="bf16", seqs=1, len_min=32768, len_max=32768, spread=False,
             heads=8, qk_heads=8, d_k=128, d_v=128, const_decay=False, states=True, reverse=False),
        # training on packed sequences of very different lengths, shared queries and keys, states passed on
        dict(name="attn_bwd_ragged_bf16", op="attn_bwd", dtype="bf16", seqs=29, len_min=1, len_max=4099, spread=True,
             heads=4, qk_heads=2, d_k=64, d_v=64, const_decay=False, states=True, reverse=False),
        # training on tracks in full precision, from the outermost hit inwards, one decay a head
        dict(name="attn_bwd_tracks_fp32", op="attn_bwd", dtype="fp32", seqs=8191, len_min=8, len_max=20,
             spread=False, heads=4, qk_heads=4, d_k=32, d_v=32, const_decay=True, states=False, reverse=True),
        # queries and keys of the tracks' layer, positions counted from each track's first hit
        dict(name="norm_tracks_bf16", op="norm", dtype="bf16", seqs=65536, len_min=8, len_max=20, spread=False,
             q_heads=3, k_heads=3, d=64, rot=64, interleaved=False, far=False),
        # training on long sequences, grouped keys, neighbouring pairs rotated
        dict(name="norm_bwd_long_bf16", op="norm_bwd", dtype="bf16", seqs=9, len_min=1024, len_max=4096,
             spread=False, q_heads=16, k_heads=4, d=128, rot=128, interleaved=True, far=False),
        # single tokens at the far end of long streams, half of each head rotated
        dict(name="norm_step_fp32", op="norm", dtype="fp32", seqs=61, len_min=1, len_max=1, spread=False,
             q_heads=8, k_heads=2, d=64, rot=32, interleaved=False, far=True),
        # single tokens of a few sequences through the block
        dict(name="ffn_tokens_bf16", op="ffn", dtype="bf16", rows=13, width=1024, inner=4096, act="silu"),
        # a training batch's forward, the largest product
        dict(name="ffn_large_bf16", op="ffn", dtype="bf16", rows=16384, width=2048, inner=5632, act="silu"),
        # a training batch's backward, odd sizes
        dict(name="ffn_bwd_odd_bf16", op="ffn_bwd", dtype="bf16", rows=5003, width=1032, inner=2731, act="gelu"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_lengths(rng, cost_per_row, budget):
    """seqs, len_min, len_max, spread within a budget of rows times cost_per_row (and of the padded square too)."""
    kind = rng.choice(["tracks", "ragged", "long"])
    rows = max(64, min(917504, int(budget / cost_per_row)))
    if kind == "tracks":
        return dict(seqs=max(1, min(65536, _log_int(rng, 16, 65536), rows // 14)), len_min=rng.randint(1, 8),
                    len_max=rng.randint(9, 20), spread=False)
    if kind == "ragged":
        hi = _log_int(rng, 65, min(4099, rows))
        return dict(seqs=max(1, min(rng.randint(2, 40), rows // hi)), len_min=1, len_max=hi, spread=True)
    n = _log_int(rng, 1024, min(32768, max(1025, rows)))
    return dict(seqs=1, len_min=n, len_max=n, spread=False)


def draw(rng):
    op = rng.choice(["step", "attn", "attn", "attn_bwd", "attn_bwd", "norm", "norm_bwd", "ffn", "ffn_bwd"])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    if op in ("step", "attn", "attn_bwd"):
        c["qk_heads"] = rng.choice([1, 2, 3, 4])
        c["heads"] = c["qk_heads"] * rng.choice([1, 1, 2, 4])
        c["d_k"], c["d_v"] = rng.choice([32, 64, 64, 128]), rng.choice([32, 64, 64, 128])
        c["const_decay"] = rng.random() < 0.3
    if op == "step":
        c["seqs"] = min(_log_int(rng, 1, 1024), (1 << 27) // (c["heads"] * c["d_k"] * c["d_v"]))
    elif op in ("attn", "attn_bwd"):
        wide = c["heads"] * max(c["d_k"], c["d_v"]) * (2 if c["dtype"] == "fp32" else 1)
        c |= _draw_lengths(rng, wide, 33554432 if op == "attn" else 12582912)
        c["states"] = rng.random() < 0.4 and c["seqs"] * c["heads"] * c["d_k"] * c["d_v"] <= 1 << 25
        c["reverse"] = rng.random() < 0.3
    elif op in ("norm", "norm_bwd"):
        c["k_heads"] = rng.choice([1, 2, 3, 4])
        c["q_heads"] = c["k_heads"] * rng.choice([1, 2, 4])
        c["d"] = rng.choice([32, 64, 128, 256])
        c["rot"] = rng.choice([c["d"], c["d"], 32, c["d"] // 2 if c["d"] > 32 else 32])
        c["interleaved"], c["far"] = rng.random() < 0.4, rng.random() < 0.3
        wide = (c["q_heads"] + c["k_heads"]) * c["d"] * (2 if c["dtype"] == "fp32" else 1)
        c |= _draw_lengths(rng, wide, 134217728 if op == "norm" else 67108864)
    else:
        c["width"] = 8 * _log_int(rng, 16, 256)
        c["inner"] = _log_int(rng, 128, 5632)
        most = 8e10 if c["dtype"] == "fp32" else 6.0e11
        rows = int(most / ((4 if op == "ffn" else 12) * c["width"] * c["inner"]))
        c["rows"] = _log_int(rng, 1, max(1, min(16384, rows)))
        c["act"] = rng.choice(["silu", "gelu"])
    return c


# ----------------------------------------------------------------------------------------------------------------
# inputs


def _lengths(case, seed):
    """The sequences' lengths: the case's own, in an order that goes by the seed (so that every seed has as many rows)."""
    lo, hi, n = case["len_min"], case["len_max"], case["seqs"]
    r = np.random.default_rng([n, lo, hi])
    if case["spread"]:
        ln = np.clip(np.exp(r.uniform(math.log(lo), math.log(hi + 1), n)).astype(np.int64), lo, hi)
    else:
        ln = r.integers(lo, hi + 1, n)
    return np.random.default_rng([seed, 11]).permutation(ln)


def _rows(case):
    return int(_lengths(case, 0).sum())


def prepare(case, seed):
    dev, t = "cuda", TYPES[case["dtype"]]
    gen = torch.Generator(device=dev)
    gen.manual_seed(1000003 * (seed + 1))

    def normal(*shape, scale=1.0, dtype=t):
        return (torch.randn(*shape, generator=gen, device=dev) * scale).to(dtype)

    s = dict(case=dict(case))
    op = case["op"]
    if op in ("attn", "attn_bwd", "step", "norm", "norm_bwd"):
        if op == "step":
            rows = case["seqs"]
        else:
            ln = _lengths(case, seed)
            off = np.zeros(len(ln) + 1, dtype=np.int32)
            off[1:] = np.cumsum(ln)
            rows, s["longest"] = int(off[-1]), int(ln.max())
            s["offsets"] = torch.from_numpy(off).to(dev)
    if op in ("attn", "attn_bwd", "step"):
        h, hk, dk, dv = case["heads"], case["qk_heads"], case["d_k"], case["d_v"]
        s["q"], s["k"], s["v"] = normal(rows, hk, dk), normal(rows, hk, dk), normal(rows, h, dv)
        # heads forget at rates between a few rows and a few hundred; the rows' own rates vary about them
        rate = 0.5 * 2.0 ** (-6.0 * torch.arange(h, device=dev, dtype=torch.float32) / max(1, h - 1))
        s["log_decay"] = -rate if case["const_decay"] else (
            -rate * torch.nn.functional.softplus(torch.randn(rows, h, generator=gen, device=dev) + 0.5))
        n = case["seqs"]
        if op == "step" or case["states"]:
            s["state"] = normal(n, h, dk, dv, dtype=torch.float32)
        if op == "attn_bwd":
            s["d_out"] = normal(rows, h, dv)
            s["d_state"] = normal(n, h, dk, dv, dtype=torch.float32) if case["states"] else None
    elif op in ("norm", "norm_bwd"):
        hq, hk, d = case["q_heads"], case["k_heads"], case["d"]
        s["q"], s["k"] = normal(rows, hq, d, scale=1.5), normal(rows, hk, d, scale=0.7)
        s["q_gain"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device=dev)
        s["k_gain"] = 1.0 + 0.2 * torch.randn(d, generator=gen, device=dev)
        s["positions"] = torch.randint(0, 1 << 20, (rows,), generator=gen, device=dev, dtype=torch.int32) \
            if case["far"] else None
        if op == "norm_bwd":
            s["d_q"], s["d_k"] = normal(rows, hq, d), normal(rows, hk, d)
    else:
        m, d, f = case["rows"], case["width"], case["inner"]
        s["x"] = normal(m, d)
        s["w_gate"], s["w_up"] = normal(f, d, scale=d ** -0.5), normal(f, d, scale=d ** -0.5)
        if op == "ffn_bwd":
            s["d_out"] = normal(m, f)
    return s


# ----------------------------------------------------------------------------------------------------------------
# the plain forms: 32 bits, rounded once at the end


def _slots(offsets, rows, padded, reverse):
    """The place of every packed row in a [seqs * padded] layout."""
    n = offsets.numel() - 1
    start, length = offsets[:-1].long(), (offsets[1:] - offsets[:-1]).long()
    ids = torch.repeat_interleave(torch.arange(n, device=offsets.device), length, output_size=rows)
    r = torch.arange(rows, device=offsets.device)
    t = start[ids] + length[ids] - 1 - r if reverse else r - start[ids]
    return ids * padded + t


def _plain_attn(q, k, v, g, s, state):
    """Linear attention with decay in chunks of at most 64 rows: products within the chunks, the chunks' states, and what the earlier
    chunks' states add.  q, k, v, state in 32 bits."""
    case, off, rows = s["case"], s["offsets"], q.shape[0]
    n, h, dk, dv = off.numel() - 1, case["heads"], case["d_k"], case["d_v"]
    c = min(64, s["longest"])
    nc = -(-s["longest"] // c)
    slots = _slots(off, rows, c * nc, case["reverse"])

    def pad(x):
        y = torch.zeros(n * c * nc, *x.shape[1:], dtype=x.dtype, device=x.device).index_copy(0, slots, x)
        return y.view(n, nc, c, *x.shape[1:])

    group = h // case["qk_heads"]
    qp = pad(q).permute(0, 3, 1, 2, 4).repeat_interleave(group, 1).contiguous()    # [n, h, nc, c, d]
    kp = pad(k).permute(0, 3, 1, 2, 4).repeat_interleave(group, 1).contiguous()
    vp = pad(v).permute(0, 3, 1, 2, 4).contiguous()
    gp = pad(g.double().expand(rows, h)).permute(0, 3, 1, 2)                       # [n, h, nc, c]
    b = gp.cumsum(-1)
    tot = b[..., -1]
    at = torch.arange(c, device=q.device)
    low = at[:, None] >= at[None, :]
    decay = torch.where(low, b[..., :, None] - b[..., None, :], torch.zeros_like(b[..., :1, None])).float().exp()
    a = torch.where(low, (qp @ kp.transpose(-1, -2)) * decay, torch.zeros_like(decay[..., :1, :1]))
    out = a @ vp
    add = (kp * (tot[..., None] - b).float().exp()[..., None]).transpose(-1, -2) @ vp
    cum = tot.cumsum(-1)                                                            # [n, h, nc]
    before = torch.arange(nc, device=q.device)
    earlier = before[:, None] > before[None, :]
    w = cum[..., :, None] - tot[..., :, None] - cum[..., None, :]
    w = torch.where(earlier, torch.where(earlier, w, torch.zeros_like(w)).float().exp(), torch.zeros_like(w[..., :1, :1]).float())
    sin = (w @ add.reshape(n, h, nc, dk * dv)).view(n, h, nc, dk, dv)
    last = ((cum[..., -1:] - cum).float().exp()[..., None, None] * add).sum(2)
    if state is not None:
        sin = sin + (cum - tot).float().exp()[..., None, None] * state[:, :, None]
        last = last + cum[..., -1].float().exp()[..., None, None] * state
    out = (out + b.float().exp()[..., None] * (qp @ sin)) * dk ** -0.5
    return out.permute(0, 2, 3, 1, 4).reshape(n * c * nc, h, dv).index_select(0, slots), last


def _plain_norm(q, k, gq, gk, s):
    case, rows = s["case"], q.shape[0]
    d, rot = case["d"], case["rot"]
    if s["positions"] is not None:
        pos = s["positions"].double()
    else:
        pos = _slots(s["offsets"], rows, 1 << 30, False).remainder(1 << 30).double()
    freq = BASE ** (-torch.arange(0, rot, 2, device=q.device, dtype=torch.float64) / rot)
    ang = pos[:, None] * freq
    co, si = ang.cos().float()[:, None], ang.sin().float()[:, None]

    def one(x, gain):
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain
        r, rest = y[..., :rot], y[..., rot:]
        if case["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack((a * co - b * si, a * si + b * co), -1).flatten(-2)
        else:
            a, b = r[..., :rot // 2], r[..., rot // 2:]
            r = torch.cat((a * co - b * si, a * si + b * co), -1)
        return torch.cat((r, rest), -1)

    return one(q, gq), one(k, gk)


def _leaf(*xs):
    return [None if x is None else x.float().requires_grad_(True) for x in xs]


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    p = 0.5 * (1 + torch.erf(g * 0.5 ** 0.5))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (2 * math.pi) ** -0.5


def _plain(s):
    case = s["case"]
    op, t = case["op"], TYPES[case["dtype"]]
    if op == "step":
        group = case["heads"] // case["qk_heads"]
        q, k = s["q"].float().repeat_interleave(group, 1), s["k"].float().repeat_interleave(group, 1)
        st = s["log_decay"].exp().expand(q.shape[0], case["heads"])[..., None, None] * s["state"] \
            + k[..., :, None] * s["v"].float()[..., None, :]
        return ((q[..., :, None] * st).sum(-2) * case["d_k"] ** -0.5).to(t), st
    if op == "attn":
        out, last = _plain_attn(s["q"].float(), s["k"].float(), s["v"].float(), s["log_decay"], s, s.get("state"))
        return (out.to(t), last) if case["states"] else out.to(t)
    if op == "attn_bwd":
        q, k, v, g, st = _leaf(s["q"], s["k"], s["v"], s["log_decay"].clone(), s.get("state"))
        out, last = _plain_attn(q, k, v, g, s, st)
        if case["states"]:
            d = torch.autograd.grad((out, last), (q, k, v, g, st), (s["d_out"].float(), s["d_state"]))
        else:
            d = torch.autograd.grad(out, (q, k, v, g), s["d_out"].float())
        return (*(x.to(t) for x in d[:3]), *d[3:])
    if op == "norm":
        q, k = _plain_norm(s["q"].float(), s["k"].float(), s["q_gain"], s["k_gain"], s)
        return q.to(t), k.to(t)
    if op == "norm_bwd":
        x = _leaf(s["q"], s["k"], s["q_gain"].clone(), s["k_gain"].clone())
        d = torch.autograd.grad(_plain_norm(*x, s), x, (s["d_q"].float(), s["d_k"].float()))
        return d[0].to(t), d[1].to(t), d[2], d[3]
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _act(g, case["act"])
    if op == "ffn":
        return (a * u).to(t)
    dh = s["d_out"].float()
    dg, du = dh * u * da, dh * a
    return (dg @ wg + du @ wu).to(t), (dg.t() @ x).to(t), (du.t() @ x).to(t)


# ----------------------------------------------------------------------------------------------------------------
# the library's calls


def _own(s):
    import paper_2609_32479_amd as tf

    case = s["case"]
    op = case["op"]
    if op == "step":
        return tf.decay_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"])
    if op == "attn":
        out, last = tf.decay_attention(s["q"], s["k"], s["v"], s["log_decay"], s["offsets"], reverse=case["reverse"],
                                       initial_state=s.get("state"), return_state=case["states"])
        return (out, last) if case["states"] else out
    if op == "attn_bwd":
        d = tf.decay_attention_backward(s["d_out"], s["q"], s["k"], s["v"], s["log_decay"], s["offsets"],
                                        reverse=case["reverse"], initial_state=s.get("state"), d_state=s["d_state"])
        return d if case["states"] else d[:4]
    if op in ("norm", "norm_bwd"):
        how = dict(offsets=s["offsets"], positions=s["positions"], rotary_dim=case["rot"], base=BASE,
                   interleaved=case["interleaved"], eps=EPS)
        if op == "norm":
            return tf.qk_norm_rotate(s["q"], s["k"], s["q_gain"], s["k_gain"], **how)
        return tf.qk_norm_rotate_backward(s["d_q"], s["d_k"], s["q"], s["k"], s["q_gain"], s["k_gain"], **how)
    if op == "ffn":
        return tf.gated_ffn(s["x"], s["w_gate"], s["w_up"], activation=case["act"])
    return tf.gated_ffn_backward(s["d_out"], s["x"], s["w_gate"], s["w_up"], activation=case["act"])


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# ----------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    op, e = case["op"], BYTES[case["dtype"]]
    if op in ("attn", "attn_bwd", "step"):
        h, hk, dk, dv = case["heads"], case["qk_heads"], case["d_k"], case["d_v"]
        rows = case["seqs"] if op == "step" else _rows(case)
        decays = 4 * h * (1 if case["const_decay"] else rows)
        state = 4 * case["seqs"] * h * dk * dv
        qkv = rows * (2 * hk * dk + h * dv) * e
        if op == "step":
            return {"bytes": qkv + rows * h * dv * e + decays + 2 * state, "flops": 5 * rows * h * dk * dv}
        # the products of a row and head: by the recurrence, or with all earlier rows where these are few
        mean = rows / case["seqs"]
        if op == "attn":
            per = min(4 * dk * dv, (mean + 1) * (dk + dv))
            return {"bytes": qkv + rows * h * dv * e + decays + (2 * state if case["states"] else 0),
                    "flops": rows * h * per}
        per = min(10 * dk * dv, (mean + 1) * (3 * dk + 2 * dv))
        return {"bytes": 2 * qkv + rows * h * dv * e + 2 * decays + (3 * state if case["states"] else 0),
                "flops": rows * h * per}
    if op in ("norm", "norm_bwd"):
        rows = _rows(case)
        vals = rows * (case["q_heads"] + case["k_heads"]) * case["d"]
        side = 4 * (rows if case["far"] else case["seqs"]) + 16 * case["d"]
        return {"bytes": (2 if op == "norm" else 3) * vals * e + side, "flops": (7 if op == "norm" else 14) * vals}
    m, d, f = case["rows"], case["width"], case["inner"]
    if op == "ffn":
        return {"bytes": (m * d + 2 * f * d + m * f) * e, "flops": 4 * m * d * f}
    return {"bytes": (2 * m * d + 4 * f * d + m * f) * e, "flops": 12 * m * d * f}


# ----------------------------------------------------------------------------------------------------------------
# 64 bits, from the definitions: the recurrences row by row


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f8 = lambda x: None if x is None else x.double()  # noqa: E731
    if op in ("ffn", "ffn_bwd"):
        x, wg, wu = f8(s["x"]), f8(s["w_gate"]), f8(s["w_up"])
        gate, up = x.matmul(wg.T), x.matmul(wu.T)
        if case["act"] == "silu":
            sg = 1 / (1 + torch.exp(-gate))
            act, der = gate * sg, sg + gate * sg * (1 - sg)
        else:
            cdf = 0.5 * torch.erfc(-gate / math.sqrt(2.0))
            act, der = gate * cdf, cdf + gate * torch.exp(-gate * gate / 2) / math.sqrt(2 * math.pi)
        if op == "ffn":
            return act * up
        d = f8(s["d_out"])
        d_gate, d_up = d * up * der, d * act
        return d_gate.matmul(wg) + d_up.matmul(wu), d_gate.T.matmul(x), d_up.T.matmul(x)
    if op in ("norm", "norm_bwd"):
        return _exact_norm(case, s)
    return _exact_attn(case, s)


def _exact_norm(case, s):
    rot, half, rows = case["rot"], case["rot"] // 2, s["q"].shape[0]
    if case["far"]:
        pos = s["positions"].double()
    else:
        o = s["offsets"].long()
        r = torch.arange(rows, device=o.device)
        pos = (r - o[torch.searchsorted(o, r, right=True) - 1]).double()
    j = torch.arange(half, device=pos.device).double()
    angle = (pos[:, None] * torch.exp(-2 * j / rot * math.log(BASE)))[:, None, :]
    co, si = torch.cos(angle), torch.sin(angle)
    first = 2 * torch.arange(half, device=pos.device) if case["interleaved"] else torch.arange(half, device=pos.device)
    second = first + (1 if case["interleaved"] else half)

    def turn(x, sign):
        y = x.clone()
        y[..., first] = co * x[..., first] - sign * si * x[..., second]
        y[..., second] = co * x[..., second] + sign * si * x[..., first]
        return y

    got, gains = [], []
    for n in "qk":
        x, gain = s[n].double(), s[n + "_gain"].double()
        inv = 1 / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + EPS)
        if case["op"] == "norm":
            got.append(turn(x * inv * gain, 1.0))
            continue
        dz = turn(s["d_" + n].double(), -1.0)
        w, hat = dz * gain, x * inv
        got.append(inv * (w - hat * (w * hat).sum(-1, keepdim=True) / case["d"]))
        gains.append((dz * hat).sum((0, 1)))
    return (*got, *gains)


def _exact_attn(case, s):
    op, h, scale = case["op"], case["heads"], case["d_k"] ** -0.5
    group = h // case["qk_heads"]
    rows = s["q"].shape[0]
    q, k = (s[n].double().repeat_interleave(group, 1) for n in "qk")
    v, g = s["v"].double(), s["log_decay"].double().expand(rows, h)
    n, dk, dv = case["seqs"], case["d_k"], case["d_v"]
    st = s["state"].double() if s.get("state") is not None else torch.zeros(n, h, dk, dv, device=q.device).double()
    if op == "step":
        st = torch.exp(g)[:, :, None, None] * st + k[:, :, :, None] * v[:, :, None, :]
        return scale * (q[:, :, None, :] @ st)[:, :, 0], st
    longest = s["longest"]
    if longest * (2 if op == "attn_bwd" else 1) > 70000 or n * h * dk * dv * longest > 3e11:
        return None
    start, length = s["offsets"][:-1].long(), s["offsets"].diff().long()
    order = torch.argsort(length, descending=True)
    alive = (length[None, :] > torch.arange(longest, device=q.device)[:, None]).sum(1).tolist()

    def row_of(t):
        """The rows of the t-th step of the sequences that are long enough, and these sequences."""
        i = order[:alive[t]]
        return (start[i] + length[i] - 1 - t if case["reverse"] else start[i] + t), alive[t]

    cur = st[order].clone()
    out = torch.empty_like(v)
    dq = torch.empty_like(q)
    do = s["d_out"].double() if op == "attn_bwd" else None
    for t in range(longest):
        r, m = row_of(t)
        cur[:m] = torch.exp(g[r])[..., None, None] * cur[:m] + k[r][..., :, None] * v[r][..., None, :]
        if op == "attn":
            out[r] = scale * (q[r][..., None, :] @ cur[:m])[..., 0, :]
        else:
            dq[r] = scale * (cur[:m] @ do[r][..., None])[..., 0]
    last = torch.empty_like(cur)
    last[order] = cur
    if op == "attn":
        return (out, last) if case["states"] else out
    # backwards: adj is the gradient of the state after the step
    dk_, dv_, dg = torch.empty_like(q), torch.empty_like(v), torch.zeros(rows, h, device=q.device).double()
    d_last = s["d_state"].double() if s["d_state"] is not None else torch.zeros_like(st)
    adj = d_last[order].clone()
    # the gradient of a row's decay: sums over the later rows of q dq - k dk, and the last state's part
    tail = (adj * cur).sum((-1, -2))
    for t in range(longest - 1, -1, -1):
        r, m = row_of(t)
        adj[:m] += scale * q[r][..., :, None] * do[r][..., None, :]
        dk_[r] = (adj[:m] @ v[r][..., None])[..., 0]
        dv_[r] = (k[r][..., None, :] @ adj[:m])[..., 0, :]
        tail[:m] += (q[r] * dq[r] - k[r] * dk_[r]).sum(-1)
        dg[r] = tail[:m]
        adj[:m] *= torch.exp(g[r])[..., None, None]
    d_first = torch.empty_like(adj)
    d_first[order] = adj
    share = lambda x: x.view(rows, case["qk_heads"], group, -1).sum(2)  # noqa: E731
    got = (share(dq), share(dk_), dv_, dg.sum(0) if case["const_decay"] else dg)
    return (*got, d_first) if case["states"] else got
