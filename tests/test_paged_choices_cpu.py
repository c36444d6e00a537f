"""What the paged attention launches, from the counts of a call alone (rt_debug_attn_choice), on both sides of
each rule; and what a model's target-only steps behind a shared prefix take (no GPU)."""
import pytest

from paper_2608_29748_amd import binding as B
from paper_2608_29748_amd.engine import config_from
from workloads import get

A16 = 1 << 20


def choose(what, heads, dtype, n_seqs, n_rows, max_rows=0, max_kv=0, window=0, sinks=0, prefix=0, ragged=False,
           max_pages=4096):
    hq, hkv, hd = heads
    kv = B.rt_paged_kv(A16, A16, A16, 8, max_pages, hkv, hd, 16, dtype)
    return B.rt_debug_attn_choice(kv, B.rt_attn_args(0, 0, 0, 0, A16 if ragged else 0, A16, n_seqs, n_rows, hq, max_rows,
                                                     max_kv, window, sinks, prefix, 0.0), what)


def test_choices_are_checked():
    for bad in (dict(what=4), dict(what=-1), dict(heads=(3, 2, 64)), dict(n_rows=0)):
        with pytest.raises(B.RetraceError) as e:
            choose(**dict(dict(what=B.RT_A_KERNEL, heads=(4, 2, 64), dtype=B.RT_BF16, n_seqs=1, n_rows=1), **bad))
        assert e.value.code == B.RT_ERR_INVALID


@pytest.mark.parametrize("heads,dtype,n_seqs,rows,kv,kernel", [
    ((32, 8, 128), B.RT_BF16, 16, 16, 300, B.RT_A_ROWS), ((32, 8, 128), B.RT_BF16, 32, 16, 700, B.RT_A_TILES),
    ((32, 8, 128), B.RT_BF16, 1, 500, 490, B.RT_A_TILES), ((32, 8, 128), B.RT_BF16, 1, 16384, 16384, B.RT_A_TILES),
    ((32, 8, 128), B.RT_BF16, 64, 1, 16384, B.RT_A_ROWS), ((32, 8, 128), B.RT_F32, 4, 4096, 4096, B.RT_A_ROWS),
    ((32, 8, 64), B.RT_F32, 64, 16, 2000, B.RT_A_ROWS_PAIRS), ((32, 8, 64), B.RT_F32, 4, 16, 2000, B.RT_A_ROWS)], ids=repr)
def test_kernels(heads, dtype, n_seqs, rows, kv, kernel):
    assert choose(B.RT_A_KERNEL, heads, dtype, n_seqs, n_seqs * rows, max_kv=kv) == kernel


@pytest.mark.parametrize("n_seqs,kv,window,kernel", [
    (8, 1016, 0, B.RT_A_ROWS), (9, 1016, 0, B.RT_A_ROWS_PAIRS), (9, 897, 0, B.RT_A_ROWS_PAIRS), (9, 896, 0, B.RT_A_ROWS),
    (9, 4000, 128, B.RT_A_ROWS), (9, 4000, 1000, B.RT_A_ROWS_PAIRS)])
def test_pairs_where_single_blocks_outnumber_the_compute_units(n_seqs, kv, window, kernel):
    """32 blocks a sequence, 256 compute units; and enough keys."""
    assert choose(B.RT_A_KERNEL, (32, 8, 64), B.RT_F32, n_seqs, n_seqs * 16, max_kv=kv, window=window) == kernel


@pytest.mark.parametrize("hd,dtype,one,parts", [(128, B.RT_BF16, 640, 641), (64, B.RT_BF16, 896, 897),
                                                (64, B.RT_F32, 640, 641), (128, B.RT_F32, 511, 512)])
def test_few_steps_are_one_part(hd, dtype, one, parts):
    for window in (0, 5000):
        n = [choose(B.RT_A_SPLITS, (8, 8, hd), dtype, 4, 4, max_kv=kv, window=window) for kv in (one, parts)]
        assert n[0] == 1 and n[1] > 1


def test_streamed_pages():
    for n, want in ((16, 0), (64, 1)):
        assert choose(B.RT_A_STREAMED, (40, 8, 128), B.RT_BF16, n, n, max_kv=4100) == want
    assert choose(B.RT_A_STREAMED, (40, 8, 128), B.RT_BF16, 64, 64 * 16, max_kv=4100) == 0     # read by several workgroups


@pytest.mark.parametrize("n,prefix,taken", [(8, 2048, False), (8, 4096, True), (64, 1024, True), (1, 16384, False),
                                            (64, 0, False)])
def test_prefix_passes(n, prefix, taken):
    splits = choose(B.RT_A_PREFIX_SPLITS, (32, 8, 128), B.RT_BF16, n, n, max_kv=prefix + 500, prefix=prefix)
    assert (splits > 0) == taken
    if taken:
        assert choose(B.RT_A_KERNEL, (32, 8, 128), B.RT_BF16, n, n, max_kv=prefix + 500, prefix=prefix) == B.RT_A_PREFIX_TILES


@pytest.mark.parametrize("n_seqs,n_rows,max_rows", [(64, 64 - 1 + 96, 96), (64, 64 - 1 + 96, 0), (64, 64, 0), (64, 64, 1),
                                                    (16, 15 + 200, 200), (64, 8, 0)])
def test_the_prefix_pass_goes_by_how_full_the_sequences_are(n_seqs, n_rows, max_rows):
    """One prompt among single tokens, or rows that nobody counted, do not take it away."""
    kw = dict(max_rows=max_rows, max_kv=8192 + 400, prefix=8192, ragged=True)
    assert choose(B.RT_A_PREFIX_SPLITS, (32, 8, 128), B.RT_BF16, n_seqs, n_rows, **kw) > 0
    assert choose(B.RT_A_KERNEL, (32, 8, 128), B.RT_BF16, n_seqs, n_rows, **kw) in (B.RT_A_PREFIX_TILES, B.RT_A_TILES)


def test_prompts_fill_tiles_by_themselves():
    for max_rows in (0, 320):
        assert choose(B.RT_A_PREFIX_SPLITS, (32, 8, 128), B.RT_BF16, 32, 32 * 208, max_rows=max_rows, max_kv=4500,
                      prefix=4096, ragged=True) == 0


@pytest.mark.parametrize("max_rows", [0, 1])
def test_steps_that_nobody_counted_are_steps(max_rows):
    kw = dict(max_rows=max_rows, max_kv=16384, window=4096, sinks=4, ragged=True)
    assert choose(B.RT_A_KERNEL, (40, 8, 128), B.RT_BF16, 64, 64, **kw) == B.RT_A_ROWS
    assert choose(B.RT_A_STREAMED, (40, 8, 128), B.RT_BF16, 64, 64, **kw) == 1


@pytest.mark.parametrize("n_seqs,prefix,taken", [(16, 1024, False), (32, 1024, False), (64, 1024, False), (16, 2048, True),
                                                 (32, 2048, True), (16, 4096, True), (4, 4096, False)])
def test_blocks_behind_a_prefix_weigh_the_parts_too(n_seqs, prefix, taken):
    splits = choose(B.RT_A_PREFIX_SPLITS, (32, 8, 128), B.RT_BF16, n_seqs, 16 * n_seqs, max_kv=prefix + 116, prefix=prefix)
    assert (splits > 0) == taken


@pytest.mark.parametrize("rows,taken", [(1, True), (3, True), (4, False), (16, False)])
def test_blocks_that_rows_fill_gain_nothing_in_fp32(rows, taken):
    """Four query heads a KV head: four rows fill a block of 16."""
    splits = choose(B.RT_A_PREFIX_SPLITS, (32, 8, 64), B.RT_F32, 64, 64 * rows, max_kv=4300, prefix=4096)
    assert (splits > 0) == taken


def step_prefix(name, seqs, prefix, positions):
    wl = get(name, batch=seqs, prompt_len=(positions, positions), new_tokens=40)
    cfg = config_from(wl.target, dtype=wl.dtype, draft_layers=wl.draft_layers, cond_layers=wl.cond_layers,
                      block_size=wl.block_size, mask_token_id=wl.mask_token_id, max_batch=seqs,
                      max_seq_len=wl.max_seq_len)
    return B.rt_debug_choice(cfg, B.RT_C_STEP_PREFIX, seqs, prefix)


@pytest.mark.parametrize("name,seqs,prefix,taken", [("tiny-f32", 64, 3600, True), ("mini-bf16", 64, 7200, True),
                                                    ("tiny-f32", 64, 0, False), ("tiny-f32", 2, 3600, False),
                                                    ("mini-bf16", 64, 160, False)])
def test_steps_behind_a_shared_prefix(name, seqs, prefix, taken):
    """The models of test_gpu_window.py's large batches make a pass over the prefix in their steps."""
    assert (step_prefix(name, seqs, prefix, max(prefix, 200) + 60) > 0) == taken


def test_shared_positions_are_checked():
    for prefix in (-16, 8, 1 << 20):
        with pytest.raises(B.RetraceError) as e:
            step_prefix("tiny-f32", 4, prefix, 200)
        assert e.value.code == B.RT_ERR_INVALID
