"""States that are infinite: given so, or past what fp32 holds.  Outputs that the recurrence makes infinite are that, with their
sign, and the others are what they are without it."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests import operator_forms as forms  # noqa: E402

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32479_amd as tf
    return tf


def _inputs(dtype, lengths, dk, dv, seed=7):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    rows, n = sum(lengths), len(lengths)
    t = {"q": r(rows, 1, dk).to(dtype), "k": r(rows, 1, dk).to(dtype), "v": r(rows, 1, dv).to(dtype), "d_out": r(rows, 1, dv).to(dtype),
         "s0": r(n, 1, dk, dv), "g": -0.05 * torch.rand(rows, 1, generator=gen)}
    return t, [0, *torch.tensor(lengths).cumsum(0).tolist()]


def _alike(name, got, want, tol):
    """Infinite in the same places with the same signs, else close in the two-norm; none is NaN."""
    got = got.double().cpu()
    assert not bool(got.isnan().any()), f"{name}: NaN"
    assert torch.equal(got.isinf(), want.isinf()), f"{name}: {int(got.isinf().sum())} infinite, not {int(want.isinf().sum())}"
    at = want.isinf()
    assert torch.equal(got[at].sign(), want[at].sign()), f"{name}: signs"
    assert forms.off(got[~at], want[~at]) <= tol, (name, forms.off(got[~at], want[~at]))


@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("dk,dv", [(32, 32), (64, 128)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_initial_state(tf, dtype, dk, dv, sign):
    t, off = _inputs(dtype, [30, 150, 9, 300], dk, dv)
    t["s0"][1, 0, 5, 17] = sign * float("inf")
    d = {k: x.double() for k, x in t.items()}
    want = forms.recurrence(d["q"], d["k"], d["v"], d["g"], off, 0.2, s0=d["s0"], d_out=d["d_out"])
    c, o = {k: x.cuda() for k, x in t.items()}, torch.tensor(off, dtype=torch.int32).cuda()
    out, last = tf.decay_attention(c["q"], c["k"], c["v"], c["g"], o, scale=0.2, initial_state=c["s0"], return_state=True)
    _alike("out", out, want["out"], forms.NORM[dtype])
    _alike("state", last, want["state"], forms.NORM_FP32)
    assert int(want["out"].isinf().sum()) == 150
    got = tf.decay_attention_backward(c["d_out"], c["q"], c["k"], c["v"], c["g"], o, scale=0.2, initial_state=c["s0"])
    _alike("dq", got[0], want["dq"], forms.NORM[dtype])


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_state_past_fp32(tf, dtype):
    """k v^T of one row overflows: the values of the state that do are infinite from there on."""
    t, off = _inputs(dtype, [30, 200, 9], 32, 64)
    t["k"][50] = 0.0
    t["v"][50] = 0.0
    t["k"][50, 0, 3], t["v"][50, 0, 40] = -1e25, 1e25
    d = {k: x.double() for k, x in t.items()}
    want = forms.recurrence(d["q"], d["k"], d["v"], d["g"], off, 0.2, s0=d["s0"])
    big = torch.finfo(FP32).max
    for n in ("out", "state"):
        want[n] = torch.where(want[n].abs() > big, want[n].sign() * float("inf"), want[n])
    want["out"] = want["out"].to(dtype).double()
    c, o = {k: x.cuda() for k, x in t.items()}, torch.tensor(off, dtype=torch.int32).cuda()
    out, last = tf.decay_attention(c["q"], c["k"], c["v"], c["g"], o, scale=0.2, initial_state=c["s0"], return_state=True)
    # the rows of the chunk with that row have it as a pair of rows, (q k) v, which may be within fp32 or past it: rows 94 to 127
    # are in the next chunk, the sequence's last ones behind a border of spans or chunks
    for rows in (slice(0, 50), slice(128, 239)):
        _alike("out", out[rows], want["out"][rows], forms.NORM[dtype])
    _alike("state", last, want["state"], forms.NORM_FP32)
