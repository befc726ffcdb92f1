"""Outputs and workspaces that are each other or an input: refused, as workgroups would write over one another's results
(made-up addresses, no GPU needed)."""
import ctypes
import os

import pytest

pytest.importorskip("torch")

A = [0x100000 * (i + 1) for i in range(16)]   # made-up device addresses, aligned and apart
BIG = 1 << 40


@pytest.fixture(scope="module")
def tf():
    import paper_2609_32479_amd as tf
    if not os.path.exists(tf.LIB_PATH):
        pytest.skip("library not built")
    return tf


def _refused(tf, call, names, pairs):
    """call(addresses by name) is refused for every pair of names with one address."""
    for a, b in pairs:
        at = dict(zip(names, A))
        at[b] = at[a]
        assert call(at) == tf.TF_EINVAL, (a, b)


def _pairs(outputs, inputs):
    return [(a, b) for i, a in enumerate(outputs) for b in outputs[:i]] + [(i, o) for o in outputs for i in inputs]


def test_decay_attention(tf):
    c = ctypes.byref(tf.DecayConfig(0, 2, 2, 32, 32, 0, 0.5))
    names = ["q", "k", "v", "g", "off", "s0", "ws", "out", "sf"]
    _refused(tf, lambda p: tf.lib().tf_decay_attention(c, p["q"], 64, p["k"], 64, p["v"], 64, p["g"], 2, 100, p["off"], 3, p["s0"], p["ws"],
                                                       BIG, p["out"], 64, p["sf"], None, None),
             names, _pairs(["ws", "out", "sf"], ["q", "k", "v", "g", "s0"]))


def test_decay_attention_backward(tf):
    c = ctypes.byref(tf.DecayConfig(0, 2, 2, 32, 32, 0, 0.5))
    names = ["do", "q", "k", "v", "g", "off", "s0", "ds", "ws", "dq", "dk", "dv", "dg", "ds0"]
    _refused(tf, lambda p: tf.lib().tf_decay_attention_backward(
        c, p["do"], 64, p["q"], 64, p["k"], 64, p["v"], 64, p["g"], 2, 100, p["off"], 3, p["s0"], p["ds"], p["ws"], BIG, p["dq"], 64,
        p["dk"], 64, p["dv"], 64, p["dg"], p["ds0"], None, None),
        names, _pairs(["ws", "dq", "dk", "dv", "dg"], ["do", "q", "k", "v", "g"]) + [("dq", "ds0"), ("dg", "ds0"), ("ws", "ds0")])


def test_decay_attention_step(tf):
    c = ctypes.byref(tf.DecayConfig(0, 2, 2, 32, 32, 0, 0.5))
    names = ["q", "k", "v", "g", "s", "s1", "out"]
    _refused(tf, lambda p: tf.lib().tf_decay_attention_step(c, p["q"], 64, p["k"], 64, p["v"], 64, p["g"], 2, 3, p["s"], p["s1"], p["out"], 64,
                                                            None),
             names, _pairs(["s1", "out"], ["q", "k", "v", "g"]) + [("s", "out")])


def test_qk_norm_rotate_backward(tf):
    c = ctypes.byref(tf.QKNormConfig(0, 2, 2, 32, 32, 0, 1e-6, 1e4))
    names = ["do", "dp", "q", "k", "gq", "gk", "ws", "dq", "dk", "dgq", "dgk"]
    _refused(tf, lambda p: tf.lib().tf_qk_norm_rotate_backward(
        c, p["do"], 64, p["dp"], 64, p["q"], 64, p["k"], 64, 100, p["gq"], p["gk"], None, None, 0, p["ws"], BIG, p["dq"], 64, p["dk"], 64,
        p["dgq"], p["dgk"], None),
        names, _pairs(["ws", "dq", "dk", "dgq", "dgk"], ["q", "k", "gq", "gk"]) + [("do", "dk"), ("dp", "dq"), ("do", "ws"), ("dp", "dgk")])


def test_gated_ffn_backward(tf):
    c = ctypes.byref(tf.GatedConfig(0, 64, 40, 0))
    names = ["do", "x", "wg", "wu", "ws", "dx", "dwg", "dwu"]
    _refused(tf, lambda p: tf.lib().tf_gated_ffn_backward(c, p["do"], 40, p["x"], 64, 100, p["wg"], p["wu"], 64, p["ws"], BIG, p["dx"], 64,
                                                          p["dwg"], p["dwu"], 64, None),
             names, _pairs(["ws", "dx", "dwg", "dwu"], ["do", "x", "wg", "wu"]))
