"""What the recurrence, the word scores and dropout refuse, through the C ABI on the host: every refusal comes before anything is launched."""
import ctypes
import math

import pytest

from paper_1809_00832_amd import binding

P = 1 << 20                 # stands for a device address; never read on these paths
OK, EINVAL, ELIMIT = binding.TL_OK, binding.TL_EINVAL, binding.TL_ELIMIT


def recurrence(**change):
    v = dict(dtype=binding.TL_DT_F32, gate=binding.TL_GATE_SIGMOID, n_trees=2, n_rows=50, channels=70, off=P, g=P, x=P, g_row=70, x_row=70)
    v.update(change)
    return binding.tl_recurrence(**v)


def workspace(r, backward=0):
    n = ctypes.c_int64(-1)
    return binding.lib().tl_recur_workspace(ctypes.byref(r) if r else None, backward, ctypes.byref(n)), n.value


Q = P + (1 << 28)           # ... and for others


def forward(r, h0=P, h=Q, h_row=70, h_last=P, tape=P, ws=P, size=1 << 40):
    return binding.lib().tl_recur(ctypes.byref(r) if r else None, h0, h, h_row, h_last, tape, ws, size, None)


def backward(r, tape=P, d_h=P, d_h_row=70, d_last=P, d_g=Q, d_g_row=70, d_x=Q + 4096, d_x_row=70, d_h0=Q, ws=P, size=1 << 40):
    return binding.lib().tl_recur_backward(ctypes.byref(r) if r else None, tape, d_h, d_h_row, d_last, d_g, d_g_row, d_x, d_x_row, d_h0, ws, size, None)


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(dtype=3), dict(gate=-1), dict(gate=2), dict(n_trees=-1), dict(n_rows=-1), dict(n_rows=(1 << 31) - (1 << 16)),
                                    dict(channels=0), dict(channels=-4), dict(channels=(1 << 20) + 1), dict(off=None), dict(g=None), dict(x=None), dict(g=P + 2), dict(x=P + 1),
                                    dict(dtype=binding.TL_DT_BF16, x=P + 1), dict(g_row=-70), dict(x_row=-1), dict(n_trees=0), dict(n_trees=1 << 23, channels=1),
                                    dict(n_trees=1 << 22, channels=1 << 20)])
def test_recurrence_refuses(change):
    r = recurrence(**change)
    row = max(70, r.channels)
    assert workspace(r)[0] == EINVAL and workspace(r, 1)[0] == EINVAL
    assert forward(r, h_row=row) == EINVAL and backward(r, d_h_row=row, d_g_row=row, d_x_row=row) == EINVAL


@pytest.mark.parametrize("change", [dict(h=None), dict(h=P + 2), dict(h_row=69), dict(h_row=0), dict(h_row=-70), dict(h0=P + 2), dict(h_last=P + 1), dict(tape=P + 2),
                                    dict(h=P)])
def test_recurrence_outputs(change):
    assert forward(recurrence(), **change) == EINVAL


@pytest.mark.parametrize("change", [dict(tape=None), dict(tape=P + 2), dict(d_h=P + 1), dict(d_h_row=-1), dict(d_last=P + 2), dict(d_g=None), dict(d_x=None), dict(d_g=P + 2),
                                    dict(d_g_row=69), dict(d_x_row=0), dict(d_h0=P + 3),
                                    dict(d_g=P), dict(d_x=P), dict(d_g=Q + 4096), dict(d_h=Q), dict(d_last=Q)])
def test_recurrence_gradients(change):
    assert backward(recurrence(), **change) == EINVAL


def test_recurrence_without_arguments():
    assert workspace(None)[0] == EINVAL and forward(None) == EINVAL and backward(None) == EINVAL
    assert binding.lib().tl_recur_workspace(ctypes.byref(recurrence()), 0, None) == EINVAL


def test_recurrence_workspace():
    few = recurrence(n_trees=1, n_rows=100000)
    for back, call in ((0, forward), (1, backward)):
        code, n = workspace(few, back)
        assert code == OK and n > 0
        assert call(few, size=n - 1) == ELIMIT and call(few, ws=None) == EINVAL and call(few, ws=P + 8) == EINVAL
        assert workspace(recurrence(), back) == (OK, 0)


def test_recurrences_that_would_be_too_large():
    """2^22 workgroups, of which a sentence has one for every 64 (fp32) or 128 channels."""
    for change, code in ((dict(n_trees=(1 << 22) - 1, channels=1), OK), (dict(n_trees=1 << 22, channels=1), EINVAL), (dict(n_trees=1 << 16, channels=4096), EINVAL),
                         (dict(n_trees=(1 << 16) - 1, channels=4096), OK), (dict(n_trees=1 << 16, channels=4096, dtype=binding.TL_DT_F16), OK),
                         (dict(n_trees=1 << 17, channels=4096, dtype=binding.TL_DT_BF16), EINVAL)):
        r = recurrence(**change)
        assert workspace(r)[0] == workspace(r, 1)[0] == code, change
        if code == EINVAL:
            assert forward(r, h_row=4096) == EINVAL and backward(r, d_h_row=4096, d_g_row=4096, d_x_row=4096) == EINVAL


def test_recurrence_with_nothing_to_do():
    r = recurrence(n_trees=0, n_rows=0, off=None, g=None, x=None)
    assert workspace(r) == (OK, 0) and forward(r, h=None) == OK and backward(r, tape=None, d_g=None, d_x=None) == OK


def score(**change):
    v = dict(dtype=binding.TL_DT_F32, n_rows=300, vocab=100, logits=P, row=100, word=P, n_top=3, logprob=P, stats=P, top_word=P, top_logprob=P, ws=None, size=0, stream=None)
    v.update(change)
    return binding.lib().tl_score(*v.values())


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(dtype=3), dict(n_rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(logits=None), dict(logits=P + 2),
                                    dict(dtype=binding.TL_DT_F16, logits=P + 1), dict(row=-100), dict(word=None), dict(word=P + 2), dict(n_top=-1), dict(n_top=65),
                                    dict(logprob=P + 1), dict(stats=P + 2), dict(top_word=None), dict(top_logprob=None), dict(top_word=P + 2), dict(top_logprob=P + 3)])
def test_scores_refuse(change):
    assert score(**change) == EINVAL


def score_backward(**change):
    v = dict(dtype=binding.TL_DT_F32, n_rows=300, vocab=100, logits=P, row=100, word=P, stats=P, d_logprob=P, d_entropy=P, d_logits=P, d_row=100, stream=None)
    v.update(change)
    return binding.lib().tl_score_backward(*v.values())


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(dtype=3), dict(n_rows=-1), dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(logits=None), dict(logits=P + 2), dict(row=-1),
                                    dict(word=None), dict(word=P + 2), dict(stats=None), dict(stats=P + 1), dict(d_logprob=P + 2), dict(d_entropy=P + 1), dict(d_logits=None),
                                    dict(d_logits=P + 2), dict(d_row=99), dict(d_row=0), dict(d_row=-100), dict(d_row=200)])
def test_gradient_of_scores_refuses(change):
    assert score_backward(**change) == EINVAL


def test_scores_workspace():
    def need(n, V, top):
        size = ctypes.c_int64(-1)
        return binding.lib().tl_score_workspace(binding.TL_DT_F32, n, V, top, ctypes.byref(size)), size.value

    code, n = need(1, 100000, 5)
    assert code == OK and n > 0
    one = dict(n_rows=1, vocab=100000, row=100000)
    assert score(**one, ws=P, size=n - 1) == ELIMIT and score(**one, ws=None, size=n) == EINVAL and score(**one, ws=P + 8, size=n) == EINVAL
    assert need(300, 100, 64) == (OK, 0) and need(0, 100, 0) == (OK, 0) and need(100000, 100000, 64) == (OK, 0)
    for bad in ((-1, 100, 0), (1, 0, 0), (1, (1 << 30) + 1, 0), (1, 100, 65), (1, 100, -1)):
        assert need(*bad)[0] == EINVAL
    assert binding.lib().tl_score_workspace(3, 1, 100, 0, ctypes.byref(ctypes.c_int64())) == EINVAL
    assert binding.lib().tl_score_workspace(0, 1, 100, 0, None) == EINVAL


def test_scores_of_no_rows():
    assert score(n_rows=0, logits=None, word=None, logprob=None, stats=None, top_word=None, top_logprob=None) == OK
    assert score_backward(n_rows=0, logits=None, word=None, stats=None, d_logits=None) == OK


def dropout(**change):
    v = dict(dtype=binding.TL_DT_F32, n_rows=3, n_cols=100, x=P, x_row=100, residual=Q, residual_row=100, y=P, y_row=100, p=0.1, numbers=P, stream=None)
    v.update(change)
    return binding.lib().tl_dropout(*v.values())


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(dtype=3), dict(n_rows=-1), dict(n_cols=0), dict(n_cols=(1 << 30) + 1), dict(x=None), dict(x=P + 2), dict(x_row=-1),
                                    dict(residual=P + 1), dict(residual_row=-5), dict(y=None), dict(y=P + 2), dict(y_row=99), dict(y_row=0), dict(p=-0.1), dict(p=1.1),
                                    dict(p=math.nan), dict(y_row=200), dict(x_row=0), dict(y=Q, residual_row=0), dict(numbers=None), dict(numbers=P + 4), dict(dtype=binding.TL_DT_BF16, y=P + 1)])
def test_dropout_refuses(change):
    assert dropout(**change) == EINVAL


def test_dropout_of_no_rows():
    assert dropout(n_rows=0, x=None, y=None, residual=None, numbers=None) == OK
