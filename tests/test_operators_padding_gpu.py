"""Rows outside of all sequences, as the rows of a static buffer that a batch does not fill: zeros in what the calls allocate, also
where that memory held NaN before, and untouched in the caller's tensors."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32479_amd as tf
    return tf


def _used_memory():
    """Blocks of many sizes full of NaN, given back to the allocator."""
    x = [torch.full((n,), float("nan"), device="cuda") for n in (64, 1000, 5000, 40000, 300000, 2000000) for _ in range(6)]
    del x


@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("qk", [1, 2])
@pytest.mark.parametrize("rows,off", [(3000, [500, 520, 520, 1300]), (70, [0, 20, 33]), (50, [50, 50]), (2500, [2400, 2500]), (40, [7])])
def test_decay_attention_in_padded_buffers(tf, dtype, qk, rows, off):
    h, dk, dv = 2, 32, 64
    r = lambda *s: torch.randn(*s, device="cuda").to(dtype)  # noqa: E731
    q, k, v, d = r(rows, qk, dk), r(rows, qk, dk), r(rows, h, dv), r(rows, h, dv)
    g, o = -torch.rand(rows, h, device="cuda"), torch.tensor(off, dtype=torch.int32, device="cuda")
    lo, hi = off[0], off[-1]
    for x in (q, k, v, d, g):   # what the padding holds is not looked at
        x[:lo], x[hi:] = float("nan"), float("nan")
    mark = lambda x: torch.full_like(x, -7.0)  # noqa: E731
    _used_memory()
    new = tf.decay_attention(q, k, v, g, o)[:1] + tf.decay_attention_backward(d, q, k, v, g, o)[:4]
    given = (tf.decay_attention(q, k, v, g, o, out=mark(v))[0],
             *tf.decay_attention_backward(d, q, k, v, g, o, dq=mark(q), dk=mark(k), dv=mark(v), d_log_decay=mark(g))[:4])
    mixed = tf.decay_attention_backward(d, q, k, v, g, o, dk=mark(k))[:4]
    for x, y in zip(new, given):
        assert torch.equal(x[lo:hi], y[lo:hi]) and bool(torch.isfinite(x).all())
        assert not bool(x[:lo].any()) and not bool(x[hi:].any())
        assert bool((y[:lo] == -7).all()) and bool((y[hi:] == -7).all())
    assert torch.equal(mixed[1], given[2]) and all(torch.equal(mixed[i], new[i + 1]) for i in (0, 2, 3))


@pytest.mark.parametrize("dtype", [BF16, FP32, FP16])
@pytest.mark.parametrize("d,rot,inter", [(32, 32, False), (128, 48, True)])
@pytest.mark.parametrize("rows,off", [(3000, [500, 520, 520, 1300]), (70, [0, 20, 33]), (50, [50, 50]), (40, [7])])
def test_norm_rotate_in_padded_buffers(tf, dtype, d, rot, inter, rows, off):
    r = lambda *s: torch.randn(*s, device="cuda").to(dtype)  # noqa: E731
    q, k, dq, dk = r(rows, 3, d), r(rows, 2, d), r(rows, 3, d), r(rows, 2, d)
    gain, o = torch.rand(d, device="cuda") + 0.5, torch.tensor(off, dtype=torch.int32, device="cuda")
    lo, hi = off[0], off[-1]
    for x in (q, k, dq, dk):
        x[:lo], x[hi:] = float("nan"), float("nan")
    mark = lambda x: torch.full_like(x, -7.0)  # noqa: E731
    how = dict(offsets=o, rotary_dim=rot, interleaved=inter)
    _used_memory()
    back = tf.qk_norm_rotate_backward(dq, dk, q, k, gain, gain, **how)
    new = (*tf.qk_norm_rotate(q, k, gain, gain, **how), *back[:2])
    other = tf.qk_norm_rotate_backward(dq, dk, q, k, gain, gain, dq=mark(q), dk=mark(k), **how)
    given = (*tf.qk_norm_rotate(q, k, gain, gain, q_out=mark(q), k_out=mark(k), **how), *other[:2])
    for x, y in zip(new, given):
        assert torch.equal(x[lo:hi], y[lo:hi]) and bool(torch.isfinite(x).all())
        assert not bool(x[:lo].any()) and not bool(x[hi:].any())
        assert bool((y[:lo] == -7).all()) and bool((y[hi:] == -7).all())
    assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(back[2:], other[2:]))
    mixed = tf.qk_norm_rotate(q, k, gain, gain, k_out=mark(k), **how)
    assert torch.equal(mixed[0], new[0]) and torch.equal(mixed[1], given[1])
