"""Tensors that require a gradient: the forward calls, which record none, refuse them where gradients are enabled, and take them
where they are not; the backward calls take them as the values that they are."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tf():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_32479_amd as tf
    return tf


def _calls(tf):
    r = lambda *s: torch.randn(*s, device="cuda")  # noqa: E731
    x = {n: r(40, 2, 32) for n in ("q", "k", "v")}
    one = {n: r(3, 2, 32) for n in ("q", "k", "v")}
    o = torch.tensor([0, 7, 40], dtype=torch.int32, device="cuda")
    return {
        "decay_attention": (tf.decay_attention, {**x, "log_decay": -torch.rand(40, 2, device="cuda"), "initial_state": r(2, 2, 32, 32)},
                            {"offsets": o}),
        "decay_attention_step": (tf.decay_attention_step, {**one, "log_decay": -torch.rand(2, device="cuda"), "state": r(3, 2, 32, 32)}, {}),
        "qk_norm_rotate": (tf.qk_norm_rotate, {"q": x["q"], "k": x["k"], "q_gain": r(32), "k_gain": r(32)}, {"offsets": o}),
        "gated_ffn": (tf.gated_ffn, {"x": r(40, 64), "w_gate": r(24, 64), "w_up": r(24, 64)}, {}),
    }


@pytest.mark.parametrize("which", ["decay_attention", "decay_attention_step", "qk_norm_rotate", "gated_ffn"])
def test_tensors_that_require_a_gradient(tf, which):
    f, tensors, rest = _calls(tf)[which]
    whole = lambda y: [t for t in (y if isinstance(y, tuple) else (y,)) if t is not None]  # noqa: E731
    want = whole(f(**tensors, **rest))
    for name in tensors:
        leaf = {**tensors, name: tensors[name].clone().requires_grad_(True)}
        with pytest.raises(RuntimeError, match=f"{name} requires"):
            f(**leaf, **rest)
        with torch.no_grad():
            assert all(torch.equal(a, b) for a, b in zip(whole(f(**leaf, **rest)), want))
        with torch.inference_mode():
            assert all(torch.equal(a, b) for a, b in zip(whole(f(**leaf, **rest)), want))
        assert all(torch.equal(a, b) for a, b in zip(whole(f(**{**leaf, name: leaf[name].detach()}, **rest)), want))


def test_weights_with_gradients_set_by_hand(tf):
    """A training step's part: the forward call without a graph, the gradients from the backward call."""
    x, d = torch.randn(90, 64, device="cuda"), torch.randn(90, 24, device="cuda")
    w = [torch.nn.Parameter(torch.randn(24, 64, device="cuda")) for _ in range(2)]
    with torch.no_grad():
        tf.gated_ffn(x, *w)
    dx, w[0].grad, w[1].grad = tf.gated_ffn_backward(d, x, *w)
    a, b = (x.double() @ p.detach().double().T for p in w)
    s = torch.sigmoid(a)
    for got, want in ((w[0].grad, (d * b * (s * (1 + a * (1 - s)))).T @ x.double()), (w[1].grad, (d * a * s).T @ x.double())):
        # fp32 sums over 64 and 90 products and the activation's dozen roundings: under 200 of 2^-24 of their magnitudes
        assert (got.double() - want).norm() <= 200 * 2.0 ** -24 * want.norm() * 8
