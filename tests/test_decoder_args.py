"""What the decoder's operators refuse, through the C ABI on the host: every refusal comes before anything is launched."""
import ctypes
import math

import pytest

from paper_1809_00832_amd import binding

P = 1 << 20                 # stands for a device address; never read on these paths
OK, EINVAL, ELIMIT = binding.TL_OK, binding.TL_EINVAL, binding.TL_ELIMIT


def rows(heads, d, p=P, row=None, head=None):
    return binding.tl_rows(p, heads * d if row is None else row, d if head is None else head)


def attention(**change):
    v = dict(dtype=binding.TL_DT_F32, n_trees=2, n_q=3, n_kv=50, n_heads=4, n_kv_heads=2, head_dim=64, scale=0.125, q_off=P, kv_off=P, kv_mask=None,
             q=rows(4, 64), k=rows(2, 64), v=rows(2, 64))
    v.update(change)
    return binding.tl_attention(**v)


def workspace(a, backward=0):
    n = ctypes.c_int64(-1)
    return binding.lib().tl_attend_workspace(ctypes.byref(a), backward, ctypes.byref(n)), n.value


def attend(a, o=None, lse=None, ws=P, size=1 << 40):
    return binding.lib().tl_attend(ctypes.byref(a), ctypes.byref(o or rows(4, 64)), lse, ws, size, None)


def backward(a, lse=P, ws=P, size=1 << 40, **change):
    v = dict(o=rows(4, 64), d_o=rows(4, 64), d_q=rows(4, 64), d_k=rows(2, 64), d_v=rows(2, 64))
    v.update(change)
    r = {k: ctypes.byref(x) if x is not None else None for k, x in v.items()}
    return binding.lib().tl_attend_backward(ctypes.byref(a), r["o"], lse, r["d_o"], r["d_q"], r["d_k"], r["d_v"], ws, size, None)


BAD = [dict(dtype=-1), dict(dtype=3), dict(n_trees=-1), dict(n_q=-1), dict(n_kv=-1), dict(n_heads=0), dict(n_heads=5), dict(n_heads=8192),
       dict(n_kv_heads=0), dict(n_kv_heads=3), dict(head_dim=0), dict(head_dim=257), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf),
       dict(scale=math.nan), dict(q_off=None), dict(kv_off=None), dict(q=rows(4, 64, p=None)), dict(k=rows(2, 64, p=None)),
       dict(v=rows(2, 64, p=None)), dict(q=rows(4, 64, p=P + 2)), dict(dtype=binding.TL_DT_F16, k=rows(2, 64, p=P + 1)),
       dict(k=rows(2, 64, row=-128)), dict(v=rows(2, 64, head=-64)), dict(n_trees=0)]


@pytest.mark.parametrize("change", BAD)
def test_attention_refuses(change):
    a = attention(**change)
    assert workspace(a)[0] == EINVAL and attend(a) == EINVAL and backward(a) == EINVAL


@pytest.mark.parametrize("o", [rows(4, 64, p=None), rows(4, 64, p=P + 1), rows(4, 64, row=0), rows(4, 64, head=0), rows(4, 64, head=63),
                               rows(4, 64, row=200), rows(4, 64, row=64, head=128), rows(4, 64, row=-256)])
def test_outputs_that_overlap_themselves(o):
    assert attend(attention(), o=o) == EINVAL
    assert backward(attention(), d_q=o) == EINVAL


def test_missing_arguments():
    assert binding.lib().tl_attend(None, ctypes.byref(rows(4, 64)), None, None, 0, None) == EINVAL
    assert binding.lib().tl_attend(ctypes.byref(attention()), None, None, None, 0, None) == EINVAL
    for name in ("o", "d_o", "d_q", "d_k", "d_v"):
        assert backward(attention(), **{name: None}) == EINVAL
    assert backward(attention(), lse=None) == EINVAL
    assert binding.lib().tl_attend_workspace(ctypes.byref(attention()), 0, None) == EINVAL


def test_workspace_is_checked():
    code, n = workspace(attention(), 1)
    assert code == OK and n >= 4 * 3 * 4
    assert backward(attention(), size=n - 1) == ELIMIT
    assert backward(attention(), ws=None) == EINVAL and backward(attention(), ws=P + 4) == EINVAL
    few = attention(n_trees=1, n_q=1, n_kv=100000)            # one query over a long axis: parts that a second launch joins
    code, n = workspace(few)
    assert code == OK and n > 0
    assert attend(few, size=n - 1) == ELIMIT and attend(few, ws=None) == EINVAL and attend(few, ws=P + 8) == EINVAL
    code, n = workspace(attention(n_trees=100, n_q=100, n_kv=1000))
    assert code == OK and n == 0


def test_nothing_to_do_is_accepted():
    a = attention(n_trees=0, n_q=0, n_kv=0, q_off=None, kv_off=None, q=rows(4, 64, p=None), k=rows(2, 64, p=None), v=rows(2, 64, p=None))
    assert workspace(a) == (OK, 0) and attend(a, o=rows(4, 64, p=None)) == OK and backward(a) == OK
    a = attention(n_q=0, q=rows(4, 64, p=None))
    assert attend(a, o=rows(4, 64, p=None), ws=None, size=0) == OK


def sample(**change):
    v = dict(dtype=binding.TL_DT_F32, n_rows=3, vocab=100, logits=P, row=100, u=P, temperature=None, top_k=None, top_p=None, min_p=None, token=P,
             logprob=None, kept=None, stream=None)
    v.update(change)
    return binding.lib().tl_sample(*v.values())


@pytest.mark.parametrize("change", [dict(dtype=-1), dict(dtype=3), dict(n_rows=-1), dict(vocab=0), dict(vocab=-5), dict(vocab=(1 << 30) + 1),
                                    dict(logits=None), dict(logits=P + 2), dict(dtype=binding.TL_DT_BF16, logits=P + 1), dict(u=None), dict(token=None),
                                    dict(row=-100)])
def test_sampling_refuses(change):
    assert sample(**change) == EINVAL


def test_sampling_no_rows():
    assert sample(n_rows=0, logits=None, u=None, token=None) == OK


LIMIT = (1 << 24) - 1       # workgroups of 256 threads in a launch


def test_launches_that_would_be_too_large():
    """2^32 threads and more: refused before anything is enqueued, also where only the second launch of a call would be too large."""
    def both(n, code, **change):
        a = attention(n_trees=n, **change)
        assert workspace(a)[0] == code and workspace(a, 1)[0] == code
        if code == EINVAL:
            assert attend(a) == EINVAL and backward(a) == EINVAL

    for n in (LIMIT // 2 + 1, LIMIT, 1 << 30, (1 << 31) - 1):                # a tree has a workgroup of its own for each of two heads
        both(n, EINVAL, n_q=n, n_kv=n)
    both(LIMIT // 4 - 8, OK, n_q=3, n_kv=50)
    assert workspace(attention(n_trees=LIMIT // 2, n_q=3))[0] == OK         # (a backward pass has both kinds of workgroups)
    # many rows of one tree: forward tiles of 128 are still few enough, the backward pass's first launch has a workgroup for 16 row heads
    a = attention(n_trees=1, n_q=1 << 26, n_kv=1)
    assert workspace(a)[0] == OK
    assert workspace(a, 1)[0] == EINVAL and backward(a) == EINVAL
    # no rows at all, a mask: one workgroup per tree
    for n in (1 << 24, (1 << 31) - 1):
        a = attention(n_trees=n, n_q=0, n_kv=0, kv_mask=P, q=rows(4, 64, p=None), k=rows(2, 64, p=None), v=rows(2, 64, p=None))
        assert backward(a) == EINVAL


@pytest.mark.parametrize("name", ["n_q", "n_kv"])
@pytest.mark.parametrize("mask", [None, P])
def test_rows_whose_numbers_would_pass_32_bits(name, mask):
    """The kernels' place in a list of nodes runs past its end by up to 2^15 before it is bounded."""
    few = dict(n_trees=1, n_q=1, n_kv=1, n_heads=1, n_kv_heads=1, head_dim=1, kv_mask=mask, q=rows(1, 1), k=rows(1, 1), v=rows(1, 1))
    most = (1 << 31) - 1 - (1 << 16)
    one = dict(o=rows(1, 1), d_o=rows(1, 1), d_q=rows(1, 1), d_k=rows(1, 1), d_v=rows(1, 1))
    for n in (most + 1, (1 << 31) - 1):
        a = attention(**dict(few, **{name: n}))
        assert workspace(a)[0] == EINVAL and workspace(a, 1)[0] == EINVAL and attend(a, o=rows(1, 1)) == EINVAL and backward(a, **one) == EINVAL
    assert workspace(attention(**dict(few, n_kv=most)))[0] == OK and workspace(attention(**dict(few, n_kv=most)), 1)[0] == OK


def test_scale_in_base_2():
    """The kernels multiply scores by scale * log2(e): where that is infinite a score of zero would be a NaN."""
    assert workspace(attention(scale=2.3e38))[0] == OK
    for scale in (2.4e38, 3.4e38):
        a = attention(scale=scale)
        assert workspace(a)[0] == EINVAL and attend(a) == EINVAL and backward(a) == EINVAL


def test_assembly_names_m0_as_written():
    import glob
    import os
    import re
    found = 0
    for path in glob.glob(os.path.join(os.path.dirname(binding.__file__), "csrc", "*.h*")):
        with open(path) as f:
            for statement in re.findall(r"asm volatile\((.*?)\);", f.read(), re.S):
                if re.search(r"s_mov_b32 m0|s_add_u32 m0", statement):
                    found += 1
                    assert '"m0"' in statement, (path, statement)
    assert found
