"""Operands of the paged-cache operators that a call cannot serve as asked, refused without a GPU."""
import pytest
import torch

from paper_2608_29748_amd import binding as B
from paper_2608_29748_amd import ops


def paged(n=4, h=2, d=64, dtype=torch.bfloat16, seqs=2, width=2):
    return (torch.zeros(n, h, 16, d, dtype=dtype), torch.zeros(n, h, d, 16, dtype=dtype),
            torch.zeros(seqs, width, dtype=torch.int32))


def refusal(call, *a, **kw):
    with pytest.raises(B.RetraceError) as e:
        call(*a, **kw)
    assert e.value.code == B.RT_ERR_INVALID
    return str(e.value)


@pytest.mark.parametrize("which", ["q", "k", "v", "q_norm", "k_norm", "q_out", "rope"])
def test_gradients_are_not_lost_silently_by_an_append(which):
    c, n = ops.PagedKV(*paged()), torch.zeros(2, dtype=torch.int32)
    t = dict(q=torch.zeros(2, 2, 64), k=torch.zeros(2, 2, 64), v=torch.zeros(2, 2, 64), q_norm=torch.ones(64).bfloat16(),
             k_norm=torch.ones(64).bfloat16(), q_out=torch.zeros(2, 2, 64).bfloat16(), rope=torch.zeros(2, 32, 32))

    def call():
        ops.kv_append(c, t["k"], t["v"], n, q=t["q"], q_out=t["q_out"], rope=t["rope"], q_norm=t["q_norm"],
                      k_norm=t["k_norm"])

    assert "not on a GPU" in refusal(call)
    t[which].requires_grad_(True)
    assert "gradient" in refusal(call)
    with torch.no_grad():
        assert "not on a GPU" in refusal(call)       # (served, on a GPU)


@pytest.mark.parametrize("which", ["q", "out"])
def test_gradients_are_not_lost_silently_by_attention(which):
    c, n = ops.PagedKV(*paged()), torch.zeros(2, dtype=torch.int32)
    t = dict(q=torch.zeros(2, 2, 64).bfloat16(), out=torch.zeros(2, 2, 64).bfloat16())
    calls = (lambda: ops.window_attention(c, t["q"], n, 16, out=t["out"]), lambda: ops.prefix_attention(c, t["q"], n, 16, out=t["out"]))
    for call in calls:
        assert "not on a GPU" in refusal(call)
    t[which].requires_grad_(True)
    for call in calls:
        assert "gradient" in refusal(call)
        with torch.no_grad():
            assert "not on a GPU" in refusal(call)


def test_caches_that_require_gradients():
    for i in (0, 1):
        t = list(paged())
        t[i].requires_grad_(True)
        assert "gradient" in refusal(ops.PagedKV, *t)
        with torch.no_grad():
            ops.PagedKV(*t)


@pytest.mark.parametrize("scale", [1e-40, 1e-46, 1e-60])
def test_a_scale_that_float32_loses_is_not_the_default(scale):
    """The C entry sees a denormal number or, from Python, what would have become 0."""
    c, n, q = ops.PagedKV(*paged()), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, 64).bfloat16()
    assert "scale" in refusal(ops.window_attention, c, q, n, 16, scale=scale)
    assert "scale" in refusal(ops.prefix_attention, c, q, n, 16, scale=scale)
    assert "not on a GPU" in refusal(ops.window_attention, c, q, n, 16, scale=2.0 ** -126)
    if scale > 1e-45:
        kv = B.rt_paged_kv(1 << 20, 1 << 20, 1 << 20, 4, 2, 2, 64, 16, B.RT_BF16)
        g = B.rt_attn_args(1 << 20, 128, 1 << 20, 128, 0, 1 << 20, 2, 2, 2, 0, 0, 16, 0, 0, scale)
        assert "scale" in refusal(B.rt_window_attention, kv, g)


def test_one_head_has_no_head_stride():
    """Rows of a single head, however the dimension of size one came about."""
    c, n = ops.PagedKV(*paged(h=1)), torch.zeros(2, dtype=torch.int32)
    one = torch.zeros(2, 64, 1).bfloat16().transpose(1, 2)
    assert one.stride(1) != 64
    assert "not on a GPU" in refusal(ops.kv_append, c, one, one, n, q=one)
    assert "not on a GPU" in refusal(ops.window_attention, c, one, n, 16, out=one.clone(memory_format=torch.preserve_format))
    assert "one after the other" in refusal(ops.window_attention, c, torch.zeros(2, 64, 2).bfloat16().transpose(1, 2), n, 16)
