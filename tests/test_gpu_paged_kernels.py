"""Every kernel of the paged attention against 64-bit results where it can go wrong: windows and sinks
around its key chunks, places that no row sees, values that are not finite, pages outside the pool,
ragged and strided rows.  Each case names the kernel that its counts lead to, and is refused if a
rule leads it elsewhere (rt_debug_attn_choice); bounds as in test_gpu_paged_bits.py."""
import math

import pytest
import torch

from paged_ref import Case
from paper_2608_29748_amd import binding as B
from test_gpu_paged_bits import BF, DEV, F32, reference, run, small_scores

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2608_29748_amd import ops
    return ops


def choice(c, what, window=0, sinks=0, prefix=0, max_rows=None, max_kv=None, uniform=False):
    kv = B.rt_paged_kv(1 << 20, 1 << 20, 1 << 20, c.n_pages, c.width, c.hkv, c.hd, 16, 1 if c.dtype == BF else 0)
    g = B.rt_attn_args(0, 0, 0, 0, 0 if c.start is None else 1 << 20, 1 << 20, len(c.rows), c.n, c.hq,
                       max(c.rows) if max_rows is None else max_rows, max(c.keys) if max_kv is None else max_kv,
                       window, sinks, prefix, 0.0)
    return B.rt_debug_attn_choice(kv, g, what)


def reach(c, kernel, streamed=0, splits=None, prefix_splits=False, **kw):
    assert choice(c, B.RT_A_KERNEL, **kw) == kernel
    assert choice(c, B.RT_A_STREAMED, **kw) == streamed
    assert (choice(c, B.RT_A_PREFIX_SPLITS, **kw) > 0) == prefix_splits
    if splits is not None:
        assert choice(c, B.RT_A_SPLITS, **kw) == splits
    return c


def check(got, ref, tol, free=()):
    """Within the bounds; NaN and infinities where the reference has NaN and nowhere else.  free: rows of
    no sequence, not looked at."""
    got = got.double()
    wild = torch.isnan(ref)
    bad = torch.where(wild, torch.isfinite(got), ~((got - ref).abs() <= tol))
    bad[list(free)] = False
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist())


def compare(ops, c, window=0, sinks=0, prefix=0, wild=(), **kw):
    """One call against the reference, its outputs in strided rows between sentinels.  wild: (sequence,
    position, element of V or None for the key itself) that hold no finite number: the rows that see
    one give none there, or nowhere."""
    kp, vp = c.kp, c.vp                        # (a weight of zero times NaN is none of the reference's)
    c.kp, c.vp = (torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (kp, vp))
    ref, tol = reference(c, window, sinks)
    c.kp, c.vp = kp, vp
    for s, j, d in wild:
        for o in range(len(c.rows)):           # (the place may be another sequence's too)
            if j // 16 < c.width and int(c.table[o, j // 16]) == int(c.table[s, j // 16]):
                p0 = c.keys[o] - c.rows[o]
                for i in range(c.rows[o]):
                    p = p0 + i
                    if j <= p and (not window or j > p - window or j < sinks):
                        ref[c.first(o) + i, :, slice(None) if d is None else d] = math.nan
    pad = 24 if c.dtype == BF else 12
    full = torch.full((c.n, c.hq * c.hd + pad), 7.0, dtype=c.dtype, device=DEV)
    out = full[:, :c.hq * c.hd].unflatten(1, (c.hq, c.hd))
    free = range(sum(c.rows), c.n)
    assert run(ops, c, window, sinks, prefix, out=out, **kw) is out
    check(out, ref, tol, free)
    assert (full[:, c.hq * c.hd:] == 7).all() and (full[sum(c.rows):] == 7).all()


def junk(c, window, sinks, value):
    """Puts `value` wherever no row of any sequence looks (keys of sequences apart)."""
    for s, n in enumerate(c.rows):
        lo = max(sinks, c.keys[s] - n - window + 1) if window else 0
        if n == 0:
            lo = c.keys[s]
        for j in range(sinks if n else 0, lo):
            page, slot = c.place(s, j)
            c.kp[page, :, slot] = value
            c.vp[page, :, :, slot] = value
    return c


# 128-row tiles over chunks of 64 keys: more than 40e6 places read by blocks of 16 rows
TILES = [((32, 8, 128), [700, 1, 0, 650, 617], [790, 300, 40, 650, 680]), ((32, 16, 64), [1310, 1, 0, 1330, 1290], [1400, 300, 40, 1330, 1350])]


@gpu
@pytest.mark.parametrize("shape", [0, 1], ids=["128", "64"])
@pytest.mark.parametrize("window,sinks", [(63, 1), (64, 0), (65, 4), (64, 63), (100, 64), (129, 65), (193, 130)])
def test_tiles_around_the_window(ops, shape, window, sinks):
    heads, rows, keys = TILES[shape]
    c = Case(rows, keys, heads, BF, seed=window, extra_rows=2, q_pad=8)
    reach(c, B.RT_A_TILES, window=window, sinks=sinks)
    compare(ops, c, window, sinks)


@gpu
@pytest.mark.parametrize("shape", [0, 1], ids=["128", "64"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_tiles_and_what_no_row_sees(ops, shape, value):
    """Behind the last key, between sinks and window, after a row's own position, in free pages; and values
    that some rows see and others do not."""
    heads, rows, keys = TILES[shape]
    window, sinks = 70, 3
    c = junk(small_scores(Case(rows, keys, heads, BF, seed=5, fill=value)), window, sinks, value)
    reach(c, B.RT_A_TILES, window=window, sinks=sinks)
    compare(ops, c, window, sinks)
    wild = [(0, keys[0] - 5, 7), (0, keys[0] - 100, 0), (3, 65, heads[2] - 1), (4, keys[4] - 130, 33), (4, 1, 2)]
    for s, j, d in wild:
        page, slot = c.place(s, j)
        c.vp[page, :, d, slot] = value
    compare(ops, c, window, sinks, wild=wild)


@gpu
@pytest.mark.parametrize("shape", [0, 1], ids=["128", "64"])
def test_tiles_and_pages_outside_the_pool(ops, shape):
    heads, rows, keys = TILES[shape]
    c = Case(rows, keys, heads, BF, seed=6)
    c.table[0, 0], c.table[0, 9], c.table[3, 20], c.table[4, keys[4] // 16 - 1] = -7, c.n_pages, 1 << 30, -1
    reach(c, B.RT_A_TILES, window=90, sinks=20)
    compare(ops, c, 90, 20)
    compare(ops, c)


@gpu
@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 16, 64)], ids=repr)
def test_tiles_of_uniform_rows(ops, heads):
    n = 16 if heads[2] == 128 else 32
    c = Case([130] * n, [130 + 9 * s for s in range(n)], heads, BF, seed=3, ragged=False)
    reach(c, B.RT_A_TILES, window=100, sinks=5)
    compare(ops, c, 100, 5)


@gpu
@pytest.mark.parametrize("heads", [(32, 8, 128), (32, 16, 64)], ids=repr)
def test_tiles_in_key_splits(ops, heads):
    """A long table: tiles whose parts a merge joins, most of them without a key."""
    c = Case([200, 3], [420, 200], heads, BF, seed=3, max_pages=512, extra_rows=1)
    reach(c, B.RT_A_TILES, window=5000, sinks=70, max_kv=8192)
    assert choice(c, B.RT_A_SPLITS, window=5000, sinks=70, max_kv=8192) > 2
    compare(ops, c, 5000, 70, max_kv=8192)
    compare(ops, c, max_kv=8192)


@gpu
@pytest.mark.parametrize("heads,rows", [((32, 8, 128), [500, 12]), ((64, 16, 64), [430, 12])], ids=repr)
@pytest.mark.parametrize("window,sinks", [(360, 0), (350, 65), (0, 0)])
def test_tiles_of_a_few_workgroups(ops, heads, rows, window, sinks):
    """A workgroup or less a compute unit, and rows at positions below 0, which see nothing."""
    c = Case(rows, [490, 12 + 300], heads, BF, seed=window, extra_rows=2)
    kw = dict(max_kv=490)
    reach(c, B.RT_A_TILES, window=window, sinks=sinks, **kw)
    compare(ops, c, window, sinks, **kw)


# fp32, head_dim 64, more than 256 blocks of 16 rows and more than 896 keys: two blocks a workgroup
@gpu
@pytest.mark.parametrize("ragged", [True, False])
@pytest.mark.parametrize("window,sinks", [(897, 0), (900, 3), (929, 33), (5000, 0)])
def test_pairs_of_row_blocks(ops, ragged, window, sinks):
    rows = [(7 * s) % 31 for s in range(12)] if ragged else [16] * 12
    c = Case(rows, [r + (197 * s) % 1100 for s, r in enumerate(rows)], (32, 8, 64), F32, seed=window, ragged=ragged,
             extra_rows=2 * ragged)
    reach(c, B.RT_A_ROWS_PAIRS, window=window, sinks=sinks)
    compare(ops, c, window, sinks)


@gpu
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_pairs_and_what_no_row_sees(ops, value):
    rows = [16 + s % 3 for s in range(12)]
    keys = [r + (197 * s) % 1100 for s, r in enumerate(rows)]
    window, sinks = 890, 3
    c = junk(small_scores(Case(rows, keys, (32, 8, 64), F32, seed=2, fill=value)), window, sinks, value)
    reach(c, B.RT_A_ROWS_PAIRS, window=window, sinks=sinks)
    compare(ops, c, window, sinks)
    wild = [(s, keys[s] - 1 - s % 20, s % 64) for s in range(0, 12, 3)] + [(5, 1, 3), (5, 95, 9), (4, 40, 60)]
    for s, j, d in wild:
        page, slot = c.place(s, j)
        c.vp[page, :, d, slot] = value
    c.table[8, 0] = c.table[10, 30] = -1
    compare(ops, c, window, sinks, wild=wild)


@gpu
def test_pairs_behind_a_prefix(ops):
    rows = [16 + s % 3 for s in range(20)]
    keys = [912 + r + s % 40 for s, r in enumerate(rows)]
    keys[5] = 900
    c = Case(rows, keys, (32, 8, 64), F32, seed=4, shared=912, extra_rows=2)
    c.table[5, :57] = c.table[0, :57]
    reach(c, B.RT_A_ROWS_PAIRS, prefix=912)         # (sixteen rows fill blocks: no pass of the prefix's own)
    compare(ops, c, prefix=912)


# pages by non-temporal loads: more than 512 MB of them, as far as the host knows
@gpu
@pytest.mark.parametrize("heads,dtype", [((16, 8, 128), BF), ((32, 8, 64), F32)], ids=repr)
@pytest.mark.parametrize("ragged", [True, False])
def test_streamed_steps(ops, heads, dtype, ragged):
    rows = [s % 3 for s in range(64)] if ragged else [1] * 64
    keys = [r + (97 * s) % 700 for s, r in enumerate(rows)]
    c = small_scores(Case(rows, keys, heads, dtype, seed=1, ragged=ragged, max_pages=256, extra_rows=ragged))
    kw = dict(max_kv=4096)
    reach(c, B.RT_A_ROWS, streamed=1, window=3000, sinks=4, **kw)
    compare(ops, c, 3000, 4, **kw)
    wild = [(s, keys[s] - 1, s % 64) for s in range(1, 64, 9)]
    for s, j, d in wild:
        page, slot = c.place(s, j)
        c.vp[page, :, d, slot] = math.nan
    compare(ops, c, wild=wild, **kw)


def shared_case(heads, dtype, seqs, each, prefix, **kw):
    rows = [each + s % 2 for s in range(seqs)]
    keys = [prefix + r + (11 * s) % 70 for s, r in enumerate(rows)]
    keys[3] = prefix - 20 + rows[3]                        # ends inside the prefix
    c = small_scores(Case(rows, keys, heads, dtype, seed=seqs, extra_rows=2, shared=prefix, **kw))
    c.table[3, :prefix // 16] = c.table[0, :prefix // 16]
    return c


# the prefix in a pass of its own: in tiles beside rows, in rows (fp32), in tiles beside tiles
@gpu
@pytest.mark.parametrize("heads,dtype,seqs,each,prefix,kernel,streamed,max_kv", [
    ((16, 8, 128), BF, 40, 1, 1600, B.RT_A_PREFIX_TILES, 0, None),
    ((16, 8, 64), BF, 60, 1, 2096, B.RT_A_PREFIX_TILES, 0, None),
    ((16, 8, 128), BF, 64, 1, 1600, B.RT_A_PREFIX_TILES, 1, 8192),
    ((16, 8, 64), BF, 64, 1, 1600, B.RT_A_PREFIX_TILES, 1, 8192),
    ((8, 4, 128), F32, 30, 2, 2080, B.RT_A_ROWS, 0, None),
    ((32, 8, 128), BF, 24, 20, 1920, B.RT_A_TILES, 0, 8192)], ids=repr)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_prefix_pass_and_values_that_are_not_finite(ops, heads, dtype, seqs, each, prefix, kernel, streamed, max_kv, value):
    c = shared_case(heads, dtype, seqs, each, prefix, fill=value, max_pages=max_kv and max_kv // 16)
    kw = dict(max_kv=max_kv or max(c.keys))
    reach(c, kernel, streamed=streamed, prefix_splits=True, prefix=prefix, **kw)
    compare(ops, c, prefix=prefix, **kw)
    # in the prefix's last page, behind what sequence 3 sees; before it; in a sequence's own keys
    wild = [(0, prefix - 2, 5), (0, prefix - 17, 9), (0, 70, 1), (2, c.keys[2] - 1, 3), (1, prefix, 2)]
    for s, j, d in wild:
        page, slot = c.place(s, j)
        c.vp[page, :, d, slot] = value
    compare(ops, c, prefix=prefix, wild=wild, **kw)


@gpu
@pytest.mark.parametrize("heads,seqs,each,prefix,kernel,max_kv", [
    ((16, 8, 128), 40, 1, 1600, B.RT_A_PREFIX_TILES, None), ((16, 8, 64), 60, 1, 2096, B.RT_A_PREFIX_TILES, None),
    ((32, 8, 128), 24, 20, 1920, B.RT_A_TILES, 8192)], ids=repr)
def test_prefix_pass_and_pages_outside_the_pool(ops, heads, seqs, each, prefix, kernel, max_kv):
    c = shared_case(heads, BF, seqs, each, prefix, max_pages=max_kv and max_kv // 16)
    c.table[:, 3], c.table[:, prefix // 16 - 1] = -1, c.n_pages + 5
    c.table[2, prefix // 16] = 1 << 30
    kw = dict(max_kv=max_kv or max(c.keys))
    reach(c, kernel, prefix_splits=True, prefix=prefix, **kw)
    compare(ops, c, prefix=prefix, **kw)


@gpu
@pytest.mark.parametrize("heads,dtype", [((16, 8, 128), BF), ((16, 8, 64), BF), ((8, 4, 128), F32)], ids=repr)
@pytest.mark.parametrize("max_rows", [0, 1, 96])
def test_one_prompt_among_tokens_behind_a_prefix(ops, heads, dtype, max_rows):
    rows = [1] * 20 + [96] + [1] * 19 + [0, 2]
    c = Case(rows, [2048 + r + (11 * s) % 70 for s, r in enumerate(rows)], heads, dtype, seed=7, extra_rows=2, shared=2048)
    assert choice(c, B.RT_A_PREFIX_SPLITS, prefix=2048, max_rows=max_rows) > 0
    compare(ops, c, prefix=2048, max_rows=max_rows)
    compare(ops, c, 300, 4, max_rows=max_rows)


@gpu
@pytest.mark.parametrize("heads,dtype,kernel", [((71, 1, 64), BF, B.RT_A_TILES), ((71, 1, 64), F32, B.RT_A_ROWS),
                                                ((96, 1, 128), BF, B.RT_A_TILES), ((96, 1, 128), F32, B.RT_A_ROWS)], ids=repr)
def test_many_heads_of_one(ops, heads, dtype, kernel):
    """More query heads of a KV head than a block or, with few rows, a tile has rows."""
    for rows, keys in (([1, 1, 0, 2], [300, 77, 5, 2]), ([900, 3, 0, 1], [950, 3, 9, 400])):
        c = Case(rows, keys, heads, dtype, seed=9, extra_rows=1)
        if rows[0] > 1:
            reach(c, kernel, window=150, sinks=2, max_kv=1000)
        compare(ops, c, 150, 2)
        compare(ops, c)


def test_the_comparison_sees_what_is_missing():
    """On the host: NaN that should be there and is not, NaN that should not, a number out of bounds."""
    ref, tol = torch.zeros(4, 2, 3, dtype=torch.float64), torch.full((4, 2, 3), 0.1, dtype=torch.float64)
    ref[1, 0, 2] = math.nan
    got = ref.float()
    check(got, ref, tol)
    got[1, 0, 2] = math.inf
    check(got, ref, tol)
    for i, x in ((1, 0.0), (2, math.nan), (2, math.inf), (3, 0.2)):
        wrong = ref.float()
        wrong[i, 0, 2] = x
        with pytest.raises(AssertionError):
            check(wrong, ref, tol)
        if i == 3:
            check(wrong, ref, tol, free=[3])
