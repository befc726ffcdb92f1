"""The sequence-layer operators' refusals, made before anything touches a GPU: the C entries' argument checks
with made-up addresses, and the binding's checks of tensors."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

A = 0x10000   # a made-up device address, aligned
B, C, D, E, F, G, H, I, J = (A + 0x1000 * i for i in range(1, 10))   # and others


@pytest.fixture(scope="module")
def tf():
    import paper_2609_32479_amd as tf
    if not os.path.exists(tf.LIB_PATH):
        pytest.skip("library not built")
    return tf


def _decay(tf, elem=1, heads=4, qk=2, dk=64, dv=32, reverse=0, scale=0.125):
    return tf.DecayConfig(elem, heads, qk, dk, dv, reverse, scale)


def _attn(tf, cfg, rows=100, qs=128, vs=128, os_=128, gs=4, n=3, off=D, ws=E, wb=1 << 40, q=A, out=F, s0=None, sf=None):
    return tf.lib().tf_decay_attention(ctypes.byref(cfg) if cfg is not None else None, q, qs, B, 128, C, vs, G, gs, rows, off,
                                       n, s0, ws, wb, out, os_, sf, None, None)


def test_decay_attention_refusals(tf):
    ok = _decay(tf)
    assert _attn(tf, ok, n=0) == tf.TF_OK                             # no sequences: nothing to do
    assert _attn(tf, None) == tf.TF_EINVAL
    for bad in (dict(elem=3), dict(heads=0), dict(qk=0), dict(qk=3), dict(dk=0), dict(reverse=2), dict(scale=float("nan")),
                dict(scale=float("inf"))):
        assert _attn(tf, _decay(tf, **bad), n=0) == tf.TF_EINVAL, bad
    for bad in (dict(dk=48), dict(dk=256), dict(dv=16), dict(heads=2048, qk=1)):
        assert _attn(tf, _decay(tf, **bad), qs=1 << 20, vs=1 << 20, os_=1 << 20, gs=0) == tf.TF_EUNSUPPORTED, bad
    for bad in (dict(rows=-1), dict(n=-1), dict(qs=127), dict(qs=132), dict(vs=120), dict(os_=64), dict(gs=3), dict(gs=-4),
                dict(off=None), dict(ws=None), dict(ws=A + 16), dict(wb=10), dict(q=None), dict(q=A + 2), dict(out=None),
                dict(out=A + 8), dict(out=A), dict(out=B), dict(out=C), dict(out=G), dict(s0=H, sf=H), dict(s0=F),
                dict(s0=H + 4), dict(sf=H + 4)):
        assert _attn(tf, ok, **bad) == tf.TF_EINVAL, bad
    assert _attn(tf, ok, rows=2 ** 31 - 1) == tf.TF_EUNSUPPORTED
    assert _attn(tf, ok, qs=(1 << 24) + 8) == tf.TF_EUNSUPPORTED
    assert _attn(tf, ok, n=2 ** 31 - 1) == tf.TF_EUNSUPPORTED
    L = tf.lib()
    assert L.tf_decay_workspace_size(ctypes.byref(ok), 100) > 0
    assert L.tf_decay_workspace_size(ctypes.byref(ok), -1) == 0
    assert L.tf_decay_workspace_size(ctypes.byref(_decay(tf, dk=48)), 100) == 0
    a = L.tf_decay_backward_workspace_size(ctypes.byref(ok), 100, 3, 0)
    assert 0 < a < L.tf_decay_backward_workspace_size(ctypes.byref(ok), 100, 3, 1)
    assert L.tf_decay_backward_workspace_size(ctypes.byref(ok), 100, -3, 1) == 0


def test_decay_backward_and_step_refusals(tf):
    L, c = tf.lib(), _decay(tf)

    def back(rows=100, ds=128, n=3, wb=1 << 40, dg=J, dq=G, d_out=A, s0=None, d_s=None, d_s0=None):
        return L.tf_decay_attention_backward(ctypes.byref(c), d_out, ds, B, 128, C, 128, D, 128, E, 4, rows, A, n, s0, d_s, F,
                                             wb, dq, 128, H, 128, I, 128, dg, d_s0, None, None)
    for bad in (dict(rows=-1), dict(ds=96), dict(n=-1), dict(wb=4), dict(dg=None), dict(dq=None), dict(dq=A + 4),
                dict(d_out=None), dict(dq=A), dict(dq=B), dict(dg=E), dict(d_out=I), dict(s0=A, d_s0=A), dict(d_s=A, d_s0=A),
                dict(d_s=A + 4)):
        assert back(**bad) == tf.TF_EINVAL, bad

    def step(n=3, st=E, so=E, qs=128, gs=4, out=F):
        return L.tf_decay_attention_step(ctypes.byref(c), A, qs, B, 128, C, 128, D, gs, n, st, so, out, 128, None)
    assert step(n=0) == tf.TF_OK
    for bad in (dict(n=-1), dict(st=None), dict(so=None), dict(so=A + 4), dict(qs=64), dict(gs=2), dict(out=None),
                dict(out=C), dict(out=E), dict(so=B)):
        assert step(**bad) == tf.TF_EINVAL, bad
    assert L.tf_decay_attention_step(ctypes.byref(_decay(tf, heads=1024, qk=1)), A, 64, A, 64, A, 1 << 15, A, 0, 2 ** 31 - 1, A, A,
                                     A, 1 << 15, None) == tf.TF_EUNSUPPORTED
    assert step(n=1 << 22) == tf.TF_EUNSUPPORTED
    assert L.tf_decay_backward_workspace_size(ctypes.byref(c), 100, 2 ** 31 - 1, 0) == 0


def test_norm_refusals(tf):
    L = tf.lib()

    def cfg(elem=1, hq=4, hk=2, d=64, rot=64, inter=0, eps=1e-6, base=1e4):
        return tf.QKNormConfig(elem, hq, hk, d, rot, inter, eps, base)

    def run(c, rows=10, qs=256, ks=128, q=A, gain=C, out=E):
        return L.tf_qk_norm_rotate(ctypes.byref(c) if c is not None else None, q, qs, B, ks, rows, gain, D, None, None, 0, out, 256,
                                   F, 128, None)
    assert run(cfg(), rows=0) == tf.TF_OK
    assert run(None) == tf.TF_EINVAL
    for bad in (dict(elem=-1), dict(hq=0), dict(rot=0), dict(rot=80), dict(eps=-1.0), dict(eps=float("nan")), dict(base=0.0),
                dict(base=float("inf"))):
        assert run(cfg(**bad)) == tf.TF_EINVAL, bad
    for bad in (dict(d=48, rot=16), dict(rot=24), dict(d=512, rot=64)):
        assert run(cfg(**bad), qs=1 << 12, ks=1 << 12) == tf.TF_EUNSUPPORTED, bad
    for bad in (dict(rows=-1), dict(qs=255), dict(qs=260), dict(ks=64), dict(q=None), dict(gain=None), dict(out=A + 8),
                dict(out=B), dict(out=C), dict(out=F), dict(out=A, qs=264)):   # in place, but in other rows
        assert run(cfg(), **bad) == tf.TF_EINVAL, bad
    assert L.tf_qk_norm_workspace_size(ctypes.byref(cfg()), 10) > 0
    assert L.tf_qk_norm_workspace_size(ctypes.byref(cfg(d=48, rot=16)), 10) == 0

    def back(wb=1 << 30, ws=E, dg=I, rows=10, dq=F, dys=256):
        return L.tf_qk_norm_rotate_backward(ctypes.byref(cfg()), A, dys, B, 128, C, 256, D, 128, rows, G, G, None, None, 0, ws, wb,
                                            dq, 256, H, 128, dg, J, None)
    for bad in (dict(wb=1), dict(ws=None), dict(dg=None), dict(rows=-1), dict(dq=None), dict(dq=C), dict(dq=H), dict(dq=B),
                dict(dq=A, dys=264)):
        assert back(**bad) == tf.TF_EINVAL, bad


def test_gated_refusals(tf):
    L = tf.lib()

    def cfg(elem=1, width=128, inner=100, act=0):
        return tf.GatedConfig(elem, width, inner, act)

    def run(c, rows=10, xs=128, ws=128, os_=100, x=A, out=D):
        return L.tf_gated_ffn(ctypes.byref(c) if c is not None else None, x, xs, rows, B, C, ws, out, os_, None)
    assert run(cfg(), rows=0) == tf.TF_OK
    assert run(None) == tf.TF_EINVAL
    for bad in (dict(elem=5), dict(width=0), dict(inner=0), dict(act=2), dict(act=-1)):
        assert run(cfg(**bad)) == tf.TF_EINVAL, bad
    assert run(cfg(width=100), xs=104, ws=104) == tf.TF_EUNSUPPORTED
    assert run(cfg(), xs=(1 << 22) + 8) == tf.TF_EUNSUPPORTED
    assert run(cfg(inner=1 << 20), rows=1 << 28, os_=1 << 20) == tf.TF_EUNSUPPORTED
    assert run(cfg(), rows=(1 << 28) + 1) == tf.TF_EUNSUPPORTED
    for bad in (dict(rows=-1), dict(xs=120), dict(xs=132), dict(ws=64), dict(os_=99), dict(x=None), dict(x=A + 8), dict(out=A + 1),
                dict(out=A), dict(out=C)):
        assert run(cfg(), **bad) == tf.TF_EINVAL, bad
    assert L.tf_gated_ffn_workspace_size(ctypes.byref(cfg()), 10) >= 10 * 2 * 128 * 2
    assert L.tf_gated_ffn_workspace_size(ctypes.byref(cfg(width=4)), 10) == 0

    def back(rows=10, wb=1 << 30, dw=G, dx=F, ds=100):
        return L.tf_gated_ffn_backward(ctypes.byref(cfg()), A, ds, B, 128, rows, C, D, 128, E, wb, dx, 128, dw, H, 128, None)
    for bad in (dict(rows=-1), dict(wb=64), dict(dw=None), dict(dx=None), dict(dx=A + 4), dict(ds=64), dict(dx=A), dict(dx=B),
                dict(dw=H), dict(dw=C)):
        assert back(**bad) == tf.TF_EINVAL, bad


def test_binding_refuses_cpu_tensors(tf):
    x = torch.zeros(4, 2, 32)
    o = torch.zeros(2, dtype=torch.int32)
    g = torch.zeros(4, 2)
    with pytest.raises(ValueError, match="GPU"):
        tf.decay_attention(x, x, x, g, o)
    with pytest.raises(ValueError, match="GPU"):
        tf.decay_attention_backward(x, x, x, x, g, o)
    with pytest.raises(ValueError, match="GPU"):
        tf.decay_attention_step(x, x, x, g, torch.zeros(4, 2, 32, 32))
    with pytest.raises(ValueError, match="GPU"):
        tf.qk_norm_rotate(x, x, x[0, 0], x[0, 0])
    with pytest.raises(ValueError, match="GPU"):
        tf.gated_ffn(x[0], x[0], x[0])


def test_binding_refuses_more_sequences_than_32_bits_count(tf, monkeypatch):
    from paper_2609_32479_amd import operators
    monkeypatch.setattr(operators, "_same", lambda *a, **k: None)
    assert operators._offsets(torch.empty(9, dtype=torch.int32, device="meta"), None) == 8
    with pytest.raises(ValueError, match="sequences"):
        operators._offsets(torch.empty(2 ** 31 + 1, dtype=torch.int32, device="meta"), None)
