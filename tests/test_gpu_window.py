"""Windowed targets and shared prefixes in whole models: prompts, rounds and target-only steps with
rt_set_window and rt_prefill_prefix, against the oracle and against the same calls without them."""
import numpy as np
import pytest

from oracle import OracleModel, OracleRunner
from paper_2608_29748_amd import binding as B
from workloads import get, make_prompts, make_weights

from gpu_parity import Report, check_decisions, compare_prefill, engine_for, run_teacher_forced

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-4, "bf16": 2e-2}


def _setup(name, **over):
    wl = get(name, norm_init="perturbed", **over)
    return wl, make_weights(wl), make_prompts(wl)


@pytest.mark.parametrize("name,window,sinks", [("tiny-f32", 20, 2), ("mini-bf16", 17, 0), ("mini-bf16-ragged", 24, 4),
                                               ("mini-bf16-gqa5", 64, 1)])
def test_windowed_rounds_match_oracle(name, window, sinks):
    """Prefill KV and five rounds, end to end and stage by stage."""
    wl, W, prompts = _setup(name)
    eng = engine_for(wl, W)
    eng.set_window(window, sinks)
    R = OracleRunner(OracleModel(wl, W, window=window, sinks=sinks))
    first = eng.prefill(prompts, wl.new_tokens)
    states = [R.prefill(p, wl.new_tokens) for p in prompts]
    assert list(first) == [st.anchor for st in states]
    compare_prefill(eng, R, wl, prompts, states, TOL[wl.dtype])
    run_teacher_forced(eng, R, wl, states, 5, TOL[wl.dtype], stages={})
    eng.close()


@pytest.mark.parametrize("name,window,sinks", [("tiny-f32", 12, 1), ("mini-bf16-ragged", 33, 4)])
def test_windowed_steps_match_oracle(name, window, sinks):
    wl, W, prompts = _setup(name)
    V, tol = wl.target.vocab, TOL[wl.dtype]
    eng = engine_for(wl, W)
    eng.set_window(window, sinks)
    m = OracleModel(wl, W, window=window, sinks=sinks)
    first = eng.prefill(prompts, wl.new_tokens)
    eng.set_debug(3)
    rep, states, tok, pos = Report(), [], [int(f) for f in first], [len(p) for p in prompts]
    for p in prompts:
        states.append(m.new_state(p, wl.new_tokens))
        m.target_forward(states[-1], p, 0)
    for step in range(6):
        g_tok, n = eng.ar_steps(1)
        assert list(n) == [1] * len(prompts)
        for i, st in enumerate(states):
            ol = m.target_forward(st, [tok[i]], pos[i]).logits[-1]
            assert rep.err("ar_logits", eng.read(B.RT_T_AR_LOGITS, i, (V,), np.float32), ol) <= tol
            check_decisions(rep, ol[None], [g_tok[i, 0]], tol, f"seq {i} step {step}")
            tok[i] = int(g_tok[i, 0])
            pos[i] += 1
    eng.close()


def stream(eng, prefill, budget, spec):
    out = [[int(f)] for f in prefill()]
    while True:
        if spec:
            t, n, _ = eng.spec_round()
        else:
            t, n = eng.ar_steps(8)
        if not n.any():
            return out
        for i, o in enumerate(out):
            o.extend(int(x) for x in t[i, :n[i]])


def test_windowed_speculation_is_the_windowed_target():
    """Graph replays, eager launches, the allocation-free round and target-only steps agree; a window of
    everything is no window; the window goes away again."""
    wl, W, prompts = _setup("tiny-f32")
    eng = engine_for(wl, W)
    budget = 40
    plain = stream(eng, lambda: eng.prefill(prompts, budget), budget, True)
    eng.set_window(10, 2)
    with pytest.raises(B.RetraceError) as e:
        eng.spec_round()
    assert e.value.code == B.RT_ERR_STATE
    win = stream(eng, lambda: eng.prefill(prompts, budget), budget, True)
    assert win != plain
    assert stream(eng, lambda: eng.prefill(prompts, budget), budget, False) == win
    eng.set_debug(2)
    assert stream(eng, lambda: eng.prefill(prompts, budget), budget, True) == win
    eng.set_debug(0)
    import torch
    first = eng.prefill(prompts, budget)
    d = [torch.zeros(wl.batch, wl.block_size, dtype=torch.int32, device="cuda"),
         torch.zeros(wl.batch, dtype=torch.int32, device="cuda"), torch.zeros(wl.batch, dtype=torch.int32, device="cuda")]
    got = [int(first[0])]
    for _ in range(budget):
        B.rt_spec_round_static(eng.h, *[x.data_ptr() for x in d])
        eng.stream.synchronize()
        got.extend(d[0][0, :int(d[1][0])].tolist())
    assert got == win[0]
    eng.set_window(1 << 30)
    assert stream(eng, lambda: eng.prefill(prompts, budget), budget, True) == plain
    eng.set_window(0)
    assert stream(eng, lambda: eng.prefill(prompts, budget), budget, True) == plain
    eng.close()


def test_profiled_windowed_round():
    """rt_profile_round and rt_time_kernel see every launch of the windowed attention."""
    wl, W, prompts = _setup("mini-bf16-ragged")
    eng = engine_for(wl, W)
    eng.set_window(40, 4)
    eng.prefill(prompts, 24)
    stats, stages, *_ = eng.profile_round()
    by = {s["kind"]: s for s in stats}
    L = wl.target.n_layers
    assert by["attention"]["launches"] >= L and by["attention"]["ms"] > 0 and by["qkv_post"]["launches"] >= L
    assert eng.time_kernel(B.RT_K_ATTENTION, 3)["launches"] == by["attention"]["launches"]
    eng.close()


def test_window_refusals():
    wl, W, _ = _setup("tiny-f32")
    eng = engine_for(wl, W)
    for bad in ((-1, 0), (8, -1), (0, 3)):
        with pytest.raises(B.RetraceError) as e:
            eng.set_window(*bad)
        assert e.value.code == B.RT_ERR_INVALID
    one = np.array([1], np.int32)
    T = eng.cfg.max_seq_len
    for code, pre, own, budget in ((B.RT_ERR_INVALID, [], [one], 4), (B.RT_ERR_INVALID, one, [[]], 4),
                                   (B.RT_ERR_CAPACITY, np.ones(T, np.int32), [one], 4),
                                   (B.RT_ERR_CAPACITY, one, [one] * 2, 4), (B.RT_ERR_TOKEN, [-1], [one], 4),
                                   (B.RT_ERR_TOKEN, one, [[wl.target.vocab]], 4), (B.RT_ERR_INVALID, one, [one], 0)):
        with pytest.raises(B.RetraceError) as e:
            eng.prefill_prefix(np.asarray(pre, np.int32), [np.asarray(p, np.int32) for p in own], budget)
        assert e.value.code == code
    eng.close()


@pytest.mark.parametrize("name,prefix", [("tiny-f32", 37), ("mini-bf16-ragged", 48), ("mini-bf16-ragged", 7)])
def test_shared_prefix_rounds_match_oracle(name, prefix):
    """A batch behind a shared prefix (of whole pages, with a rest, and of no page at all): the
    cache, rounds end to end, and the same tables undone by the next prefill."""
    wl, W, prompts = _setup(name, **({"batch": 3} if name == "tiny-f32" else {}))
    pre = prompts[0][:prefix]
    own = [p[prefix:] if i == 0 else p[:20 + 9 * i] for i, p in enumerate(prompts)]
    own = [p if len(p) else prompts[1][:5] for p in own]
    full = [np.concatenate([pre, p]) for p in own]
    eng = engine_for(wl, W)
    R = OracleRunner(OracleModel(wl, W))
    first = eng.prefill_prefix(pre, own, 24)
    states = [R.prefill(p, 24) for p in full]
    assert list(first) == [st.anchor for st in states]
    compare_prefill(eng, R, wl, full, states, TOL[wl.dtype])
    run_teacher_forced(eng, R, wl, states, 3, TOL[wl.dtype], stages={})
    eng.set_debug(0)
    first = eng.prefill(prompts, 24)
    states = [R.prefill(p, 24) for p in prompts]
    assert list(first) == [st.anchor for st in states]
    compare_prefill(eng, R, wl, prompts, states, TOL[wl.dtype])
    eng.close()


@pytest.mark.parametrize("name,seqs,prefix,window", [("tiny-f32", 64, 3600, 0), ("mini-bf16", 64, 7200, 0),
                                                     ("mini-bf16", 64, 7200, 300)])
def test_a_batch_large_enough_for_the_prefix_pass(name, seqs, prefix, window):
    """64 sequences behind a long prefix, whose steps' attention is one pass over the prefix and one
    over the rest, against the same prompts prefilled apart: steps and rounds."""
    wl, W, _ = _setup(name, batch=seqs, prompt_len=(prefix + 60, prefix + 60), new_tokens=40)
    V, tol = wl.target.vocab, TOL[wl.dtype]
    g = np.random.default_rng(3)
    pre = g.integers(0, V - 1, prefix).astype(np.int32)
    own = [g.integers(0, V - 1, 1 + (7 * i) % 50).astype(np.int32) for i in range(seqs)]
    full = [np.concatenate([pre, p]) for p in own]
    apart, shared = engine_for(wl, W), engine_for(wl, W)
    if window:
        apart.set_window(window, 4)
        shared.set_window(window, 4)
    rep = Report()
    same = np.ones(seqs, bool)
    fa, fs = apart.prefill(full, 30), shared.prefill_prefix(pre, own, 30)
    same &= fa == fs
    for e in (apart, shared):
        e.set_debug(3)
    for step in range(2):
        (ta, _), (ts, _) = apart.ar_steps(1), shared.ar_steps(1)
        for i in np.nonzero(same)[0][::7]:
            la, ls = (e.read(B.RT_T_AR_LOGITS, int(i), (V,), np.float32) for e in (apart, shared))
            assert rep.err("steps", la, ls) <= tol
        same &= ta[:, 0] == ts[:, 0]
    assert same.mean() > 0.9
    for e, f in ((apart, lambda: apart.prefill(full, 30)), (shared, lambda: shared.prefill_prefix(pre, own, 30))):
        f()
    same = fa == fs
    for t in range(2):
        stats = shared.profile_round() if t == 1 else None
        if stats is not None:
            launches = {s["kind"]: s["launches"] for s in stats[0]}
            assert launches["attention"] == wl.draft_layers + wl.target.n_layers
            break
        (ta, na, _), (ts, ns, _) = apart.spec_round(), shared.spec_round()
        for i in np.nonzero(same)[0][::7]:
            la, ls = (e.read(B.RT_T_DRAFT_LOGITS, int(i), (wl.block_size, V), np.float32) for e in (apart, shared))
            assert rep.err("draft", la, ls) <= tol
            la, ls = (e.read(B.RT_T_VERIFY_LOGITS, int(i), (V,), np.float32) for e in (apart, shared))
            assert rep.err("verify", la, ls) <= tol
        assert (ta[same, 0] == ts[same, 0]).mean() > 0.9
    for e in (apart, shared):
        e.close()


@pytest.mark.parametrize("window", [0, 24])
def test_sampled_rounds_behind_a_shared_prefix(window):
    """Draws depend on the seed, the sequence and the round alone: the same tokens as apart."""
    wl, W, prompts = _setup("tiny-f32", batch=3, temperature=1.0)
    pre, own = prompts[0][:40], [p[40 + 3 * i:50 + 5 * i] for i, p in enumerate(prompts)]
    eng = engine_for(wl, W)
    if window:
        eng.set_window(window, 2)
    got = []
    for prefill in (lambda: eng.prefill([np.concatenate([pre, p]) for p in own], 40),
                    lambda: eng.prefill_prefix(pre, own, 40)):
        first = prefill()
        rounds = [eng.spec_round() for _ in range(3)]
        got.append((list(first), [[list(x[s, :n[s]]) for s in range(3)] for x, n, _ in rounds]))
    assert got[0] == got[1]
    eng.close()
