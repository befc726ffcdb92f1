"""The binding's own checks, on the CPU: tensors of the meta device stand in for the GPU's."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def operators(monkeypatch):
    from paper_2609_32479_amd import operators
    monkeypatch.setattr(operators, "_same", lambda *a, **k: None)
    monkeypatch.setattr(operators, "_elem", lambda x: 1)
    return operators


def _meta(*shape):
    return torch.empty(*shape, device="meta")


def test_sizes_past_32_bits_are_refused(operators):
    w = _meta(2 ** 32 + 5, 8)   # would count as 5 inner values
    with pytest.raises(ValueError, match="inner 4294967301"):
        operators._gated_inputs(_meta(3, 8), w, w, "silu")
    x = _meta(4, 2, 64)
    with pytest.raises(ValueError, match="rotary_dim"):
        operators._norm_inputs(x, x, _meta(64), _meta(64), None, None, 2 ** 32 + 64, 1e4, False, 1e-6, None, None)
    with pytest.raises(ValueError, match="n_q_heads"):
        operators._norm_inputs(_meta(1, 2 ** 32 + 2, 64), x[:1], _meta(64), _meta(64), None, None, 64, 1e4, False, 1e-6, None, None)
    with pytest.raises(ValueError, match="n_heads"):
        operators._decay_inputs(x[:1], x[:1], _meta(1, 2 ** 32 + 2, 32), None, False)
    assert operators._gated_inputs(_meta(3, 8), _meta(5, 8), _meta(5, 8), "silu")[0][0].inner == 5


class _Device:
    """Stands in for torch.cuda.device: counts what is entered and not left."""
    inside = 0

    def __init__(self, index):
        pass

    def __enter__(self):
        _Device.inside += 1

    def __exit__(self, *exc):
        _Device.inside -= 1


class _Tensor:
    device = "cuda:1"

    def get_device(self):
        return 1


class _Stream:
    def __init__(self, index):
        self.device, self.cuda_stream = torch.device("cuda", index), 4096


def test_streams_that_do_not_fit_leave_the_device_as_it_was(monkeypatch):
    from paper_2609_32479_amd import operators
    monkeypatch.setattr(torch.cuda, "device", _Device)
    monkeypatch.setattr(torch.cuda, "stream", _Device)
    monkeypatch.setattr(operators.torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with operators._On(_Tensor(), _Stream(1)) as handle:
        assert handle == 4096 and _Device.inside == 2
    assert _Device.inside == 0
    for stream, error in ((object(), TypeError), (_Stream(0), ValueError)):
        with pytest.raises(error):
            with operators._On(_Tensor(), stream):
                pass
        assert _Device.inside == 0


def test_heads_without_a_width_reach_the_library(operators):
    """... which refuses them with its own error."""
    import ctypes
    import os

    import paper_2609_32479_amd as tf
    x = _meta(4, 2, 0)
    (cfg, _), strides = operators._decay_inputs(x, x, _meta(4, 2, 32), None, False)
    assert (cfg.d_k, strides) == (0, (0, 0, 64))
    if os.path.exists(tf.LIB_PATH):
        assert tf.lib().tf_decay_workspace_size(ctypes.byref(cfg), 4) == 0
