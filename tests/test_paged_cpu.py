"""The paged-cache operators without a GPU: every malformed call is refused before any device
work, and the workspace follows from the counts."""
import numpy as np
import pytest
import torch

from paper_2608_29748_amd import binding as B
from paper_2608_29748_amd import ops

A16 = 1 << 20      # an aligned address that is never touched


def cache(**over):
    f = dict(k=A16, v=A16, page_table=A16, n_pages=8, max_pages=4, n_kv_heads=2, head_dim=64, page_size=16,
             dtype=B.RT_BF16)
    f.update(over)
    return B.rt_paged_kv(**f)


def append(**over):
    f = dict(q=A16, k=A16, v=A16, ldq=256, ldk=128, ldv=128, q_out=A16, ldqo=256, row_start=0, kv_len=A16, rope=A16,
             q_norm=0, k_norm=0, src_dtype=B.RT_F32, n_seqs=2, n_rows=4, n_q_heads=4, rope_positions=64, rot_dim=64,
             eps=1e-6)
    f.update(over)
    return B.rt_append_args(**f)


def attn(**over):
    f = dict(q=A16, ldq=256, out=A16, ldo=256, row_start=0, kv_len=A16, n_seqs=2, n_rows=4, n_q_heads=4, max_rows=0,
             max_kv=0, window=16, sinks=4, prefix_len=0, scale=0.0)
    f.update(over)
    return B.rt_attn_args(**f)


def refused(code, call, *args):
    with pytest.raises(B.RetraceError) as e:
        call(*args)
    assert e.value.code == code, e.value
    assert str(e.value)


BAD_CACHE = [dict(dtype=2), dict(page_size=32), dict(head_dim=96), dict(n_kv_heads=0), dict(n_pages=0),
             dict(max_pages=0), dict(max_pages=(1 << 26) + 1), dict(k=0), dict(v=0), dict(page_table=0),
             dict(k=A16 + 8), dict(v=A16 + 2), dict(page_table=A16 + 2)]


@pytest.mark.parametrize("bad", BAD_CACHE, ids=repr)
def test_bad_caches(bad):
    refused(B.RT_ERR_INVALID, B.rt_kv_append, cache(**bad), append())
    refused(B.RT_ERR_INVALID, B.rt_window_attention, cache(**bad), attn())
    assert B.rt_attn_workspace_bytes(cache(**bad), attn()) == 0 and B.rt_last_error()


@pytest.mark.parametrize("code,bad", [
    (B.RT_ERR_INVALID, dict(n_seqs=-1)), (B.RT_ERR_INVALID, dict(n_rows=-1)), (B.RT_ERR_INVALID, dict(n_seqs=0)),
    (B.RT_ERR_INVALID, dict(n_seqs=3)), (B.RT_ERR_INVALID, dict(n_q_heads=3)), (B.RT_ERR_INVALID, dict(n_q_heads=0)),
    (B.RT_ERR_CAPACITY, dict(n_rows=1 << 28)), (B.RT_ERR_INVALID, dict(kv_len=0)),
    (B.RT_ERR_INVALID, dict(kv_len=A16 + 1)), (B.RT_ERR_INVALID, dict(row_start=A16 + 2)),
    (B.RT_ERR_INVALID, dict(q=A16 + 4)), (B.RT_ERR_INVALID, dict(ldq=255)), (B.RT_ERR_INVALID, dict(ldq=258)),
], ids=repr)
def test_bad_rows(code, bad):
    refused(code, B.rt_kv_append, cache(), append(**{**bad, **({"ldq": 257} if bad.get("ldq") == 258 else {})}))
    refused(code, B.rt_window_attention, cache(), attn(**bad))
    refused(code, B.rt_prefix_attention, cache(), attn(**dict(dict(window=0, sinks=0), **bad)))


@pytest.mark.parametrize("code,bad", [
    (B.RT_ERR_INVALID, dict(src_dtype=3)), (B.RT_ERR_INVALID, dict(rot_dim=8)), (B.RT_ERR_INVALID, dict(rot_dim=24)),
    (B.RT_ERR_INVALID, dict(rot_dim=80)), (B.RT_ERR_CAPACITY, dict(rope_positions=63)),
    (B.RT_ERR_INVALID, dict(rope=A16 + 4)), (B.RT_ERR_INVALID, dict(q_norm=A16 + 2)),
    (B.RT_ERR_INVALID, dict(k_norm=A16 + 8)), (B.RT_ERR_INVALID, dict(eps=-1.0)),
    (B.RT_ERR_INVALID, dict(eps=float("nan"))), (B.RT_ERR_INVALID, dict(k=0)), (B.RT_ERR_INVALID, dict(v=0)),
    (B.RT_ERR_INVALID, dict(q_out=0)), (B.RT_ERR_INVALID, dict(ldk=64)), (B.RT_ERR_INVALID, dict(ldv=130)),
    (B.RT_ERR_INVALID, dict(ldqo=260)),
], ids=repr)
def test_bad_appends(code, bad):
    refused(code, B.rt_kv_append, cache(), append(**bad))


def test_append_of_other_source_types():
    refused(B.RT_ERR_INVALID, B.rt_kv_append, cache(dtype=B.RT_F32), append(src_dtype=B.RT_BF16))


@pytest.mark.parametrize("bad", [dict(window=0), dict(window=-1), dict(sinks=-1), dict(prefix_len=16), dict(max_rows=-1),
                                 dict(max_kv=-5), dict(scale=-1.0), dict(scale=float("inf")), dict(out=0),
                                 dict(ldo=128), dict(out=A16 + 8)], ids=repr)
def test_bad_window_calls(bad):
    refused(B.RT_ERR_INVALID, B.rt_window_attention, cache(), attn(**bad))


@pytest.mark.parametrize("bad", [dict(window=16), dict(sinks=1), dict(prefix_len=-16), dict(prefix_len=8),
                                 dict(prefix_len=80)], ids=repr)
def test_bad_prefix_calls(bad):
    refused(B.RT_ERR_INVALID, B.rt_prefix_attention, cache(), attn(**dict(dict(window=0, sinks=0), **bad)))


def test_null_structures_and_workspaces():
    for call in (B.rt_window_attention, B.rt_prefix_attention):
        refused(B.RT_ERR_INVALID, call, None, attn())
        refused(B.RT_ERR_INVALID, call, cache(), None)
    refused(B.RT_ERR_INVALID, B.rt_kv_append, None, append())
    refused(B.RT_ERR_INVALID, B.rt_kv_append, cache(), None)
    assert B.rt_attn_workspace_bytes(None, attn()) == 0
    kv, g = cache(max_pages=64), attn(window=0, sinks=0, prefix_len=512)
    need = B.rt_attn_workspace_bytes(kv, g)
    assert need > 0        # the prefix and the rest are two parts at least
    for code, ptr, size in ((B.RT_ERR_WORKSPACE, 0, need), (B.RT_ERR_WORKSPACE, A16, need - 1),
                            (B.RT_ERR_WORKSPACE, A16 + 128, need)):
        refused(code, B.rt_prefix_attention, kv, g, ptr, size)


def test_calls_without_rows_do_nothing():
    none = dict(n_rows=0, q=0, kv_len=0)
    B.rt_kv_append(cache(), append(k=0, v=0, q_out=0, **none))
    B.rt_kv_append(cache(), append(k=0, v=0, q_out=0, n_seqs=0, **none))
    B.rt_window_attention(cache(), attn(out=0, **none))
    B.rt_prefix_attention(cache(), attn(out=0, window=0, sinks=0, prefix_len=16, **none))
    assert B.rt_attn_workspace_bytes(cache(), attn(out=0, **none)) == 0


def test_more_workgroups_than_a_launch_has():
    rows = dict(n_seqs=1, n_rows=(1 << 28) - 1)
    refused(B.RT_ERR_CAPACITY, B.rt_kv_append, cache(), append(**rows))
    refused(B.RT_ERR_CAPACITY, B.rt_window_attention, cache(dtype=B.RT_F32), attn(**rows))
    refused(B.RT_ERR_CAPACITY, B.rt_prefix_attention, cache(dtype=B.RT_F32), attn(window=0, sinks=0, **rows))


def test_workspace_is_of_the_counts_alone():
    kv = cache(max_pages=4096)
    g = dict(n_seqs=3, n_rows=3, max_kv=60000, window=30000, sinks=0)
    need = B.rt_attn_workspace_bytes(kv, attn(**g))
    assert need > 0 and need == B.rt_attn_workspace_bytes(kv, attn(q=0, out=0, **g))
    assert need % 256 == 0


def paged(n=4, h=2, d=64, dtype=torch.bfloat16, seqs=2, width=2):
    return (torch.zeros(n, h, 16, d, dtype=dtype), torch.zeros(n, h, d, 16, dtype=dtype),
            torch.zeros(seqs, width, dtype=torch.int32))


def test_tensor_checks():
    k, v, t = paged()
    c = ops.PagedKV(k, v, t)
    for bad in ((k, k, t), (k, v.float(), t), (k, v, t.long()), (k.half(), v.half(), t), (k[0], v, t),
                (k, v.transpose(0, 1).contiguous().transpose(0, 1), t), (k, v, t[0])):
        refused(B.RT_ERR_INVALID, ops.PagedKV, *bad)
    n = torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(2, 2, 64, dtype=torch.bfloat16)

    def no(call, *a, **kw):
        with pytest.raises(B.RetraceError) as e:
            call(c, *a, **kw)
        assert e.value.code == B.RT_ERR_INVALID

    no(ops.kv_append, rows, rows, n.long())
    no(ops.kv_append, rows, rows, torch.zeros(3, dtype=torch.int32))
    no(ops.kv_append, rows, rows, n, row_start=n)
    no(ops.kv_append, rows, rows.float(), n)
    no(ops.kv_append, rows.half(), rows.half(), n)
    no(ops.kv_append, rows[..., :32], rows[..., :32], n)
    no(ops.kv_append, rows[:, :1], rows[:, :1], n)
    no(ops.kv_append, rows.transpose(0, 1).contiguous().transpose(0, 1), rows, n)
    no(ops.kv_append, rows, rows, n, q_out=rows)
    no(ops.kv_append, rows, rows, n, q=rows, q_out=rows.float())
    no(ops.kv_append, rows, rows, n, rope=torch.zeros(2, 32, 32).double())
    no(ops.kv_append, rows, rows, n, q_norm=torch.zeros(64))
    no(ops.window_attention, rows.float(), n, 16)
    no(ops.window_attention, rows, n, 16, out=rows.float())
    no(ops.window_attention, rows[:1].expand(2, 2, 64)[:, :, ::2], n, 16)
    no(ops.prefix_attention, rows, n, 8)
    no(ops.window_attention, rows, n, (1 << 32) + 5)
    no(ops.window_attention, rows, n, 16, 1 << 31)
    no(ops.window_attention, rows, n, 16, max_kv=-1)
    no(ops.prefix_attention, rows, n, 1 << 32)
    no(ops.prefix_attention, rows, n, 16, workspace=torch.zeros(64, 64)[:, ::2])


def test_rope_table_is_the_rounds_table():
    t = ops.rope_table(1e6, 64, 40, "cpu")
    for p in (0, 1, 39):
        for i in (0, 5, 31):
            ang = np.float32(p) * np.float32(1e6 ** (-2.0 * i / 64))
            assert t[0, p, i] == np.float32(np.cos(np.float64(ang))) and t[1, p, i] == np.float32(np.sin(np.float64(ang)))
