"""Configurations that name outputs to clear: refused where they name none that there is (no GPU needed)."""
import ctypes
import os

import pytest

pytest.importorskip("torch")


@pytest.fixture(scope="module")
def tf():
    import paper_2609_32479_amd as tf
    if not os.path.exists(tf.LIB_PATH):
        pytest.skip("library not built")
    return tf


@pytest.mark.parametrize("clear,fine", [(0, True), (1, True), (15, True), (16, False), (-1, False)])
def test_decay_clear(tf, clear, fine):
    c = ctypes.byref(tf.DecayConfig(1, 4, 2, 64, 32, 0, 0.125, clear))
    assert (tf.lib().tf_decay_workspace_size(c, 100) > 0) == fine
    none = tf.lib().tf_decay_attention(c, None, 128, None, 128, None, 128, None, 4, 0, None, 0, None, None, 0, None, 128, None, None, None)
    assert none == (tf.TF_OK if fine else tf.TF_EINVAL)


@pytest.mark.parametrize("clear,fine", [(0, True), (3, True), (4, False), (-1, False)])
def test_norm_clear(tf, clear, fine):
    c = ctypes.byref(tf.QKNormConfig(1, 4, 2, 64, 64, 0, 1e-6, 1e4, clear))
    assert (tf.lib().tf_qk_norm_workspace_size(c, 100) > 0) == fine
