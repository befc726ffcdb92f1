"""Linear attention with decay where states have to be carried: sequences of many spans whose heads forget slowly or not at
all, so that what a row gets from far away is most of it; heads that forget at once, whose decays' gradient is small against the
sums that it comes from; against the recurrence in 64 bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from tests import operator_forms as forms  # noqa: E402

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
# rows before the first and behind the last sequence, spans of 128 rows: the long sequence is cut by 23 borders
LENGTHS, START, TAIL = [3000, 1, 0, 500, 40], 300, 200


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32479_amd as tf
    return tf


def _inputs(seed, dtype, lengths, heads, qk, dk, dv, decay, start=0, tail=0):
    gen = torch.Generator().manual_seed(seed)
    off = np.concatenate(([0], np.cumsum(lengths))) + start
    rows = int(off[-1]) + tail
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    t = {"q": r(rows, qk, dk).to(dtype), "k": r(rows, qk, dk).to(dtype), "v": r(rows, heads, dv).to(dtype),
         "d_out": r(rows, heads, dv).to(dtype), "s0": r(len(lengths), heads, dk, dv), "d_state": r(len(lengths), heads, dk, dv)}
    u = torch.rand(rows, heads, generator=gen)
    t["g"] = {"slow": -1e-3 * (0.5 + u), "none": torch.zeros(rows, heads), "fast": -20.0 - u,
              "mixed": -0.6 * 4.0 ** -torch.arange(heads).float() * (0.5 + u)}[decay]
    return t, off.astype(np.int32)


def _ref(t, off, scale, reverse, states, **kw):
    d = {k: x.double() for k, x in t.items()}
    return forms.recurrence(d["q"], d["k"], d["v"], d["g"], off.tolist(), scale, reverse=reverse, s0=d["s0"] if states else None,
                            d_out=d["d_out"], d_state=d["d_state"] if states else None, **kw)


NAMES = ("out", "state", "dq", "dk", "dv", "dg", "d_initial")


def _tolerance(name, dtype):
    return forms.NORM[FP32 if name in ("state", "dg", "d_initial") else dtype]


@pytest.mark.parametrize("decay,reverse,states", [("slow", False, True), ("none", True, False), ("mixed", True, True)])
def test_the_tolerances_find_a_lost_state(decay, reverse, states):
    """A mistake in the recurrence (on the CPU): the states lost at the spans' borders, or at one of them in the middle."""
    t, off = _inputs(3, FP32, [1000, 40], 2, 1, 32, 32, decay)
    want = _ref(t, off, 0.2, reverse, states)
    for drop in (range(128, 1000, 128), (512,)):
        got = _ref(t, off, 0.2, reverse, states, drop=set(drop))
        for n in ("out", "dq", "dk", "dv", "dg"):
            assert forms.off(got[n], want[n]) > 2 * forms.NORM[BF16], (n, forms.off(got[n], want[n]))
    for n in NAMES:
        if n != "d_initial" or states:
            assert forms.off(torch.zeros_like(want[n]), want[n]) == 1.0 > _tolerance(n, BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("shape", [(2, 1, 32, 64), (2, 2, 64, 64)])
@pytest.mark.parametrize("decay,reverse,states", [("slow", False, True), ("slow", True, False), ("none", True, True),
                                                  ("none", False, False), ("mixed", False, True)])
def test_states_carried_over_many_spans(tf, dtype, shape, decay, reverse, states):
    heads, qk, dk, dv = shape
    print(f"[chains] {dtype} {shape} {decay} reverse {reverse} states {states}", flush=True)
    t, off = _inputs(31, dtype, LENGTHS, heads, qk, dk, dv, decay, START, TAIL)
    _check(tf, t, off, dtype, dk ** -0.5, reverse, states)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,shape,length,reverse", [(FP32, (1, 1, 32, 32), 9001, False), (BF16, (1, 1, 32, 32), 9001, True),
                                                        (BF16, (1, 1, 128, 128), 1500, False), (FP32, (1, 1, 128, 32), 1500, True)])
def test_states_carried_over_chains_longer_than_a_wave(tf, dtype, shape, length, reverse):
    """9001 rows: 70 borders, more than a wave's lanes; and the wide heads."""
    heads, qk, dk, dv = shape
    t, off = _inputs(37, dtype, [5, length], heads, qk, dk, dv, "slow")
    _check(tf, t, off, dtype, dk ** -0.5, reverse, True)


def _check(tf, t, off, dtype, scale, reverse, states):
    want = _ref(t, off, scale, reverse, states)
    c, o = {k: x.cuda() for k, x in t.items()}, torch.from_numpy(off).cuda()
    mark = lambda x: torch.full_like(x, -7.0)  # noqa: E731
    s0 = c["s0"] if states else None
    got = dict(zip(("out", "state"), tf.decay_attention(c["q"], c["k"], c["v"], c["g"], o, reverse=reverse, initial_state=s0,
                                                        return_state=True, out=mark(c["v"]))))
    got |= dict(zip(NAMES[2:], tf.decay_attention_backward(
        c["d_out"], c["q"], c["k"], c["v"], c["g"], o, reverse=reverse, initial_state=s0, d_state=c["d_state"] if states else None,
        dq=mark(c["q"]), dk=mark(c["k"]), dv=mark(c["v"]), d_log_decay=mark(c["g"]))))
    lo, hi = int(off[0]), int(off[-1])
    for n in NAMES:
        if n == "d_initial" and not states:
            continue
        x, w = got[n], want[n]
        if n not in ("state", "d_initial"):
            assert bool((x[:lo] == -7).all()) and bool((x[hi:] == -7).all()), f"{n}: rows outside of all sequences"
            x, w = x[lo:hi], w[lo:hi]
            if n == "dg":   # heads that forget at different rates, each for itself
                for j in range(x.shape[1]):
                    assert forms.off(x[:, j], w[:, j]) <= _tolerance(n, dtype), (n, j, forms.off(x[:, j], w[:, j]))
        assert forms.off(x, w) <= _tolerance(n, dtype), (n, forms.off(x, w), _tolerance(n, dtype))


@pytest.mark.gpu
def test_decays_gradient_over_spans_against_differences(tf):
    """One sequence that four borders cut: the loss's slope in the log decays, by central differences in 64 bits."""
    t, off = _inputs(41, FP32, [700], 2, 1, 32, 32, "mixed")
    c, o, d = {k: x.cuda() for k, x in t.items()}, torch.from_numpy(off).cuda(), {k: x.double() for k, x in t.items()}
    dg = tf.decay_attention_backward(c["d_out"], c["q"], c["k"], c["v"], c["g"], o, scale=0.2, initial_state=c["s0"],
                                     d_state=c["d_state"])[3].double().cpu()

    def loss(g):
        r = forms.recurrence(d["q"], d["k"], d["v"], g, off.tolist(), 0.2, s0=d["s0"])
        return ((r["out"] * d["d_out"]).sum() + (r["state"] * d["d_state"]).sum()).item()
    gen, h = torch.Generator().manual_seed(5), 1e-5
    for part in (slice(0, 700), slice(0, 128), slice(300, 420)):
        way = torch.zeros_like(d["g"])
        way[part] = torch.randn(way[part].shape, generator=gen).double()
        slope, mine = (loss(d["g"] + h * way) - loss(d["g"] - h * way)) / (2 * h), (dg * way).sum().item()
        # a difference is off by h^2 of third derivatives (the sums over up to 700 rows cubed: 1e-10 of 1e3), the gradient by
        # 2^-14 in its two-norm
        assert abs(slope - mine) <= 2.0 ** -12 * (dg * way).norm().item(), (part, slope, mine)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("shape", [(2, 1, 32, 32), (2, 2, 64, 64), (1, 1, 32, 128)])
@pytest.mark.parametrize("reverse", [False, True])
def test_decays_gradient_of_heads_that_forget_at_once(tf, dtype, shape, reverse):
    """Log decays near -20: a row's gradient is e^-20 of the products of pairs, and has to be good to its own size although the
    sums over rows and over columns that it is the difference of are 5e8 times larger."""
    heads, qk, dk, dv = shape
    t, off = _inputs(43, dtype, [500, 20, 1, 64, 65], heads, qk, dk, dv, "fast", 9, 5)
    want = _ref(t, off, dk ** -0.5, reverse, False)["dg"]
    c, o = {k: x.cuda() for k, x in t.items()}, torch.from_numpy(off).cuda()
    got = tf.decay_attention_backward(c["d_out"], c["q"], c["k"], c["v"], c["g"], o, reverse=reverse)[3][9:-5].double().cpu()
    # the only pairs that count are neighbours: with magnitudes m = |q| |k| |d_out| |v| e^g scale of each
    a = {k: x.double().abs() for k, x in t.items()}
    group = heads // qk
    q, k = a["q"].repeat_interleave(group, 1), a["k"].repeat_interleave(group, 1)
    one = (q[1:] * k[:-1]).sum(-1) * (a["d_out"][1:] * a["v"][:-1]).sum(-1)
    two = (q[:-1] * k[1:]).sum(-1) * (a["d_out"][:-1] * a["v"][1:]).sum(-1)
    m = float((two if reverse else one).max()) * float(torch.exp(t["g"].double().max())) * dk ** -0.5
    # Roundings of a pair: q k and d_out v (d + 2 each), the exponential's argument of 29 (two of them: 58 ln 2), two products:
    # under 4 d + 256 of 2^-24 of m.  At each of up to nine borders of chunks in a span, and at its end, the state's pairs are
    # added and taken away: at most 40 in all.  The sums' cancellation: fp64's 2^-53 of 2^8 pairs of e^20 m
    bound = 40 * (4 * max(dk, dv) + 256) * 2.0 ** -24 * m + 2.0 ** -45 * 5e8 * m
    err = (got - want[9:-5]).abs().max().item()
    print(f"[fast] {dtype} {shape} {reverse}: {err:.2e} of {bound:.2e}, largest gradient {want.abs().max().item():.2e}", flush=True)
    assert err <= bound < want.abs().max().item() / 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("reverse", [False, True])
def test_decays_gradient_of_heads_that_forget_at_once_with_states(tf, dtype, first, reverse):
    """The last states' gradients reach such a head's rows only through their last one; its own gradient is e^-20 of it."""
    dk, dv = 64, 32
    t, off = _inputs(47, dtype, [20, 1, 0, 30, 9], 1, 1, dk, dv, "fast")
    d = {k: x.double() for k, x in t.items()}
    want = forms.recurrence(d["q"], d["k"], d["v"], d["g"], off.tolist(), 0.1, reverse=reverse, s0=d["s0"] if first else None,
                            d_out=d["d_out"], d_state=d["d_state"])["dg"]
    c, o = {k: x.cuda() for k, x in t.items()}, torch.from_numpy(off).cuda()
    got = tf.decay_attention_backward(c["d_out"], c["q"], c["k"], c["v"], c["g"], o, scale=0.1, reverse=reverse,
                                      initial_state=c["s0"] if first else None, d_state=c["d_state"])[3].double().cpu()
    # The gradient's terms are e^g times two of: scale q k d_out v, k dS v, scale q S0 d_out, dS S0 (that of a sequence of one row
    # has the last); roundings as of the heads above, in one chunk
    a = {k: x.double().abs() for k, x in t.items()}
    e = float(torch.exp(t["g"].double().max()))
    pair = 0.1 * float(a["q"].sum(-1).max()) * float(a["k"].max()) * float(a["d_out"].sum(-1).max()) * float(a["v"].max())
    state = float(torch.einsum("rk,skv,rv->rs", a["k"][:, 0], a["d_state"][:, 0], a["v"][:, 0]).max())
    begin = 0.1 * float(torch.einsum("rk,skv,rv->rs", a["q"][:, 0], a["s0"][:, 0], a["d_out"][:, 0]).max()) + float(
        (a["d_state"] * a["s0"]).sum((-1, -2)).max())
    m = e * (pair + state + (begin if first else 0.0))
    bound = 2 * (4 * dk + 256) * 2.0 ** -24 * m + 2.0 ** -45 * 5e8 * m
    err = (got - want).abs().max().item()
    print(f"[fast] {dtype} {first} {reverse}: {err:.2e} of {bound:.2e}, largest gradient {want.abs().max().item():.2e}", flush=True)
    assert err <= bound < want.abs().max().item() / 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("reverse,states", [(False, False), (True, True)])
def test_gradient_of_one_decay_a_head(tf, dtype, reverse, states):
    """log_decay of one value a head: the sum of the rows' gradients over all sequences, cut ones among them."""
    t, off = _inputs(59, dtype, [900, 1, 0, 20, 65], 4, 2, 64, 32, "mixed", 5, 3)
    one = -0.6 * 4.0 ** -torch.arange(4).float()
    t["g"] = one.expand(t["g"].shape).contiguous()
    rows = _ref(t, off, 0.125, reverse, states)["dg"][off[0]:off[-1]]
    c, o = {k: x.cuda() for k, x in t.items()}, torch.from_numpy(off).cuda()
    got = tf.decay_attention_backward(c["d_out"], c["q"], c["k"], c["v"], one.cuda(), o, scale=0.125, reverse=reverse,
                                      initial_state=c["s0"] if states else None, d_state=c["d_state"] if states else None)[3].double().cpu()
    want = rows.sum(0)
    # the rows' gradients are off by NORM_FP32 in the two-norm: their sum by at most that times the root of their number
    bound = forms.NORM_FP32 * rows.norm(dim=0) * len(rows) ** 0.5
    print(f"[one decay] {dtype} {(got - want).abs().tolist()} of {bound.tolist()}, {want.tolist()}", flush=True)
    assert bool(((got - want).abs() <= bound).all()) and bool((bound < want.abs() / 4).all())
