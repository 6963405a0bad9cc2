"""Which of the feed-forward sublayer's buffers live on when a larger one takes their place, without a GPU: tensors are made in host memory."""
import gc
import weakref

import pytest
import torch

from paper_2003_00532_b200 import feed_forward


@pytest.fixture
def capturing(monkeypatch):
    """Buffers in host memory, and whether the stream is being captured: a list of one truth value."""
    state, empty = [False], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: empty(*a, **{**k, "device": "cpu"}))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state[0])
    return state


def _grown(buffers, capturing, when):
    """A reference to the buffer of one token, after a call for eight has replaced it; captured: in its first or its second use."""
    refs = []
    for use in range(2):
        capturing[0] = use in when
        buffers._begin()
        one = buffers._buffer("n", 1, 16, dtype=torch.float32)
        refs.append((weakref.ref(one._base), one.data_ptr()))
        capturing[0] = False
    assert refs[0][1] == refs[1][1]
    del one
    buffers._begin()
    eight = buffers._buffer("n", 8, 16, dtype=torch.float32)
    gc.collect()
    assert eight.shape == (8, 16)
    return refs[0][0]


def test_a_captured_buffer_outlives_its_replacement(capturing):
    for when in ((0,), (1,), (0, 1)):
        buffers = feed_forward._Buffers()
        assert _grown(buffers, capturing, when)() is not None, when
        again = buffers._buffer("n", 1, 16, dtype=torch.float32)
        assert again.data_ptr() == buffers._buffer("n", 8, 16, dtype=torch.float32).data_ptr()   # eager calls use the larger one


def test_any_other_buffer_is_given_back(capturing):
    buffers = feed_forward._Buffers()
    assert _grown(buffers, capturing, ())() is None


def test_captured_calls_keep_one_buffer_each(capturing):
    buffers = feed_forward._Buffers()
    capturing[0] = True
    buffers._begin()
    for _ in range(5):
        for tokens in (1, 3, 2):
            buffers._buffer("n", tokens, 16, dtype=torch.float32)
    assert [b.shape[0] for b in buffers._captured] == [1, 3]
