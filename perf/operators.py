"""Operators over the paged KV cache, timed apart from a model: appending keys and values
with the position rotation on the way, attention with a sliding window and sinks, and
attention for a batch whose sequences share a prefix.

The cache is the library's: K pages [page][kv head][16][head_dim] and V pages
[page][kv head][head_dim][16], found through a page table per sequence.  Sequences bring
their rows one after the other (row_start), and a sequence of n rows whose cache holds
kv_len keys, those rows' own among them, has its row i at position kv_len - n + i.

The plain forms are elementary torch operations in 32 bits on the same pages.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
PAGE = 16
THETA, EPS = 1e6, 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases

def _append(name, n_seqs, rows, ctx, heads, dtype, src, norm=True):
    """rows and ctx: ranges of a sequence's new rows and of the keys it held before."""
    return dict(name=name, op="append", n_seqs=n_seqs, rows_lo=rows[0], rows_hi=rows[1], ctx_lo=ctx[0],
                ctx_hi=ctx[1], hq=heads[0], hkv=heads[1], hd=heads[2], dtype=dtype, src=src, norm=norm)


def _window(name, n_seqs, rows, ctx, heads, dtype, window, sinks):
    return dict(name=name, op="window", n_seqs=n_seqs, rows_lo=rows[0], rows_hi=rows[1], ctx_lo=ctx[0],
                ctx_hi=ctx[1], hq=heads[0], hkv=heads[1], hd=heads[2], dtype=dtype, window=window, sinks=sinks)


def _prefix(name, n_seqs, rows, ctx, heads, dtype, prefix):
    """ctx: keys a sequence holds of its own, behind the prefix and before its new rows."""
    return dict(name=name, op="prefix", n_seqs=n_seqs, rows_lo=rows[0], rows_hi=rows[1], ctx_lo=ctx[0],
                ctx_hi=ctx[1], hq=heads[0], hkv=heads[1], hd=heads[2], dtype=dtype, prefix=prefix)


H06, H4, H14, TINY = (16, 8, 128), (32, 8, 128), (40, 8, 128), (4, 2, 64)


def listed():
    return [
        # one token of one session, straight from the fp32 projection: launch latency only
        _append("append step", 1, (1, 1), (512, 512), H06, "bf16", "f32"),
        # a batch of short prompts of unequal lengths, of a small fp32 model
        _append("append prompts f32", 8, (96, 320), (0, 0), TINY, "f32", "f32"),
        # a long prompt in the storage type, its keys and queries without a norm of their own
        _append("append prompt", 2, (8192, 16384), (0, 100), H4, "bf16", "bf16", norm=False),
        # one token of one session of a windowed model
        _window("window step", 1, (1, 1), (8192, 8192), H06, "bf16", 1024, 4),
        # a step of a full batch of long sessions: the window is what has to be read
        _window("window steps", 64, (1, 1), (4096, 16384), H14, "bf16", 4096, 4),
        # a long prompt: matrix products
        _window("window prompt", 1, (16384, 16384), (0, 0), H4, "bf16", 4096, 4),
        # short prompts of unequal lengths, of a small fp32 model
        _window("window prompts f32", 8, (17, 320), (0, 200), TINY, "f32", 128, 1),
        # a small group of samples of one prompt
        _prefix("prefix steps small", 4, (1, 1), (1, 64), H06, "bf16", 512),
        # a batch of requests under one system prompt, a token each
        _prefix("prefix steps", 64, (1, 1), (1, 1024), H4, "bf16", 8192),
        # the same verified in blocks of 16 rows, as a speculative round does
        _prefix("prefix blocks", 16, (16, 16), (96, 320), H14, "bf16", 16384),
        # short suffix prompts of unequal lengths behind a prefix, of a small fp32 model
        _prefix("prefix prompts f32", 8, (1, 60), (0, 0), TINY, "f32", 1024),
        # the suffix prompts of a batch of requests under one system prompt
        _prefix("prefix prompts", 32, (96, 320), (0, 0), H4, "bf16", 4096),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def span(lo, hi):
        a, b = log_int(lo, hi), log_int(lo, hi)
        return min(a, b), max(a, b)

    op = rng.choice(["append", "window", "prefix"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hkv = rng.choice([2, 4, 8])
    hd = rng.choice([64, 128]) if dtype == "bf16" else 64
    heads = (hkv * rng.choice([1, 2, 3, 4, 5, 8]), hkv, hd)
    n_seqs = log_int(1, 64)
    kind = rng.choice(["steps", "blocks", "prompts"])
    most = max(17, (16384 if dtype == "bf16" else 2048) // n_seqs)
    rows = (1, 1) if kind == "steps" else (16, 16) if kind == "blocks" else span(2, most)
    if op == "append":
        case = _append("", n_seqs, rows, span(1, 4096), heads, dtype,
                       "f32" if dtype == "f32" else rng.choice(["f32", "bf16"]), rng.random() < 0.5)
    elif op == "window":
        ctx = span(1, 16384 if kind != "prompts" else 2048)
        case = _window("", n_seqs, rows, ctx, heads, dtype, log_int(16, 4096), rng.choice([0, 1, 4, 16, 100]))
    else:
        case = _prefix("", n_seqs, rows, span(1, 1024), heads, dtype, PAGE * log_int(4, 512))
    del case["name"]
    while work(case)["flops"] > 9e11:       # no dearer than the longest listed prompt
        case["rows_lo"], case["rows_hi"] = max(1, case["rows_lo"] // 2), case["rows_hi"] // 2
    return case


# ------------------------------------------------------------------ inputs

def _lens(case):
    """Rows and keys (the rows' own among them) of every sequence; the case alone decides."""
    r = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    rows = [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["n_seqs"])]
    held = [r.randint(case["ctx_lo"], case["ctx_hi"]) + case.get("prefix", 0) for _ in range(case["n_seqs"])]
    return rows, [a + b for a, b in zip(held, rows)]


def prepare(case, seed):
    rows, keys = _lens(case)
    n, S = sum(rows), case["n_seqs"]
    hq, hkv, hd, dt = case["hq"], case["hkv"], case["hd"], TYPES[case["dtype"]]
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device=DEVICE) * std).to(dtype)

    # pages in no particular order; what lies behind a prefix is a sequence's own
    shared = case.get("prefix", 0) // PAGE
    need = [(k + PAGE - 1) // PAGE - shared for k in keys]
    n_pages, width = shared + sum(need) + 1, shared + max(need)
    order = np.random.default_rng(seed).permutation(n_pages)
    table = np.zeros((S, width), np.int32)
    at = shared
    for s in range(S):
        table[s, :shared] = order[:shared]
        table[s, shared:shared + need[s]] = order[at:at + need[s]]
        at += need[s]
    i32 = dict(dtype=torch.int32, device=DEVICE)
    uniform = case["rows_lo"] == case["rows_hi"]
    st = dict(op=case["op"], kp=normal(n_pages, hkv, PAGE, hd), vp=normal(n_pages, hkv, hd, PAGE),
              table=torch.from_numpy(table).to(DEVICE), kv_len=torch.tensor(keys, **i32),
              row_start=None if uniform else torch.tensor([0] + list(np.cumsum(rows)), **i32),
              max_rows=max(rows), max_kv=max(keys), n_seqs=S, hq=hq, hkv=hkv, hd=hd,
              window=case.get("window"), sinks=case.get("sinks"), prefix=case.get("prefix"))
    if case["op"] == "append":
        src = TYPES[case["src"]]
        qkv = normal(n, hq + 2 * hkv, hd, dtype=src)      # one projection's rows: strided heads
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        st["q_norm"] = st["k_norm"] = None
        if case["norm"]:
            st["q_norm"], st["k_norm"] = (1 + normal(hd, std=0.1, dtype=torch.float32)).to(dt), \
                (1 + normal(hd, std=0.1, dtype=torch.float32)).to(dt)
        inv = torch.tensor([THETA ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=torch.float32)
        ang = (torch.arange(width * PAGE, dtype=torch.float32)[:, None] * inv).double()
        st["rope"] = torch.stack([ang.cos(), ang.sin()]).float().to(DEVICE)      # [cos, sin][position][hd / 2]
        st["q_out"] = torch.zeros(n, hq, hd, dtype=dt, device=DEVICE)
    else:
        st["q"] = normal(n, hq, hd, std=1.5)
    if own:
        from paper_2608_29748_amd import ops
        st["cache"] = ops.PagedKV(st["kp"], st["vp"], st["table"])
    return st


# ------------------------------------------------------------------ one pass

def run(state):
    st = state
    if own:
        from paper_2608_29748_amd import ops
        if st["op"] == "append":
            ops.kv_append(st["cache"], st["k"], st["v"], st["kv_len"], row_start=st["row_start"], q=st["q"],
                          q_out=st["q_out"], rope=st["rope"], q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS)
            return st["q_out"], st["kp"], st["vp"]
        if st["op"] == "window":
            return ops.window_attention(st["cache"], st["q"], st["kv_len"], st["window"], st["sinks"],
                                        row_start=st["row_start"], max_rows=st["max_rows"], max_kv=st["max_kv"])
        return ops.prefix_attention(st["cache"], st["q"], st["kv_len"], st["prefix"], row_start=st["row_start"],
                                    max_rows=st["max_rows"], max_kv=st["max_kv"])
    if st["op"] == "append":
        return _plain_append(st)
    return _plain_attention(st)


def _row_start(st):
    if st["row_start"] is not None:
        return st["row_start"].long()
    return torch.arange(st["n_seqs"] + 1, device=DEVICE) * st["max_rows"]


def _plain_append(st):
    start = _row_start(st)
    row = torch.arange(st["q"].shape[0], device=DEVICE)
    seq = (row[:, None] >= start[None, 1:]).sum(1)
    pos = st["kv_len"].long()[seq] - (start[seq + 1] - row)
    cos, sin = st["rope"][0, pos][:, None], st["rope"][1, pos][:, None]
    half = st["hd"] // 2

    def turn(x, w):
        x = x.float()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    page, slot = st["table"].long()[seq, pos // PAGE], pos % PAGE
    st["q_out"].copy_(turn(st["q"], st["q_norm"]))
    st["kp"][page, :, slot] = turn(st["k"], st["k_norm"]).to(st["kp"].dtype)
    st["vp"][page, :, :, slot] = st["v"].to(st["vp"].dtype)
    return st["q_out"], st["kp"], st["vp"]


def _plain_attention(st):
    hq, hkv, hd, G = st["hq"], st["hkv"], st["hd"], st["hq"] // st["hkv"]
    n, S, T, R = st["q"].shape[0], st["n_seqs"], st["max_kv"], st["max_rows"]
    start, kv_len = _row_start(st), st["kv_len"].long()
    count = start[1:] - start[:-1]
    out = torch.zeros(n + 1, hkv, G, hd, dtype=st["q"].dtype, device=DEVICE)     # the last row takes the padding
    j = torch.arange(T, device=DEVICE)
    s_step = max(1, (1 << 28) // (T * hkv * hd))
    for s0 in range(0, S, s_step):
        s1 = min(S, s0 + s_step)
        pages = st["table"][s0:s1, :(T + PAGE - 1) // PAGE].long()
        K = st["kp"][pages].float().permute(0, 2, 4, 1, 3).reshape(s1 - s0, hkv, hd, -1)[..., :T].contiguous()
        V = st["vp"][pages].float().permute(0, 2, 1, 4, 3).reshape(s1 - s0, hkv, -1, hd)[:, :, :T].contiguous()
        r_step = max(1, (1 << 28) // ((s1 - s0) * hq * T))
        for r0 in range(0, R, r_step):
            i = torch.arange(r0, min(R, r0 + r_step), device=DEVICE)
            live = i[None] < count[s0:s1, None]
            row = torch.where(live, start[s0:s1, None] + i[None], n)
            pos = (kv_len - count)[s0:s1, None] + i[None]
            q = st["q"][row.clamp(max=n - 1)].float().reshape(s1 - s0, -1, hkv, G, hd)
            q = (q / math.sqrt(hd)).permute(0, 2, 1, 3, 4).reshape(s1 - s0, hkv, -1, hd)
            sc = torch.matmul(q, K).reshape(s1 - s0, hkv, len(i), G, T)
            seen = j <= pos[..., None]
            if st["op"] == "window":
                seen = seen & ((pos[..., None] - j < st["window"]) | (j < st["sinks"]))
            sc = sc.masked_fill(~seen[:, None, :, None], -torch.inf)
            m = sc.amax(-1, keepdim=True)
            p = torch.exp(sc - torch.where(m == -torch.inf, 0.0, m))
            den = p.sum(-1, keepdim=True)
            o = torch.matmul(p.reshape(s1 - s0, hkv, -1, T), V).reshape(s1 - s0, hkv, len(i), G, hd)
            o = torch.where(den > 0, o / den, 0.0)
            out[row] = o.permute(0, 2, 1, 3, 4).to(out.dtype)
    return out[:n].reshape(n, hq, hd)


# ------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    rows, keys = _lens(case)
    hq, hkv, hd, G = st["hq"], st["hkv"], st["hd"], st["hq"] // st["hkv"]
    table = st["table"].cpu().numpy()
    first = np.concatenate([[0], np.cumsum(rows)])
    if case["op"] == "append":
        qo, kp, vp = st["q_out"].double(), st["kp"].double(), st["vp"].double()
        turned = {}
        for name in "qk":
            x = st[name].double()
            if case["norm"]:
                x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * st[name + "_norm"].double()
            turned[name] = x
        for s in range(case["n_seqs"]):
            a, b, p0 = int(first[s]), int(first[s + 1]), keys[s] - rows[s]
            w = torch.complex(st["rope"][0, p0:keys[s]].double(), st["rope"][1, p0:keys[s]].double())
            for name in "qk":
                x = turned[name][a:b]
                z = torch.complex(x[..., :hd // 2].contiguous(), x[..., hd // 2:].contiguous()) * w[:, None]
                turned[name][a:b] = torch.cat([z.real, z.imag], -1)
            v = st["v"][a:b].double()
            for i0 in range(p0 // PAGE * PAGE, keys[s], PAGE):
                lo, hi = max(i0, p0), min(i0 + PAGE, keys[s])
                page = int(table[s, i0 // PAGE])
                kp[page, :, lo - i0:hi - i0] = turned["k"][a + lo - p0:a + hi - p0].transpose(0, 1)
                vp[page, :, :, lo - i0:hi - i0] = v[lo - p0:hi - p0].permute(1, 2, 0)
        qo.copy_(turned["q"])
        return qo, kp, vp
    out = torch.zeros(int(first[-1]), hq, hd, dtype=torch.float64, device=DEVICE)
    for s in range(case["n_seqs"]):
        pages = torch.from_numpy(table[s, :(keys[s] + PAGE - 1) // PAGE]).long().to(DEVICE)
        K = st["kp"][pages].transpose(1, 2).reshape(-1, hkv, hd)[:keys[s]].double()
        V = st["vp"][pages].permute(0, 3, 1, 2).reshape(-1, hkv, hd)[:keys[s]].double()
        step = max(1, (1 << 26) // (G * keys[s]))
        for r0 in range(0, rows[s], step):
            r1 = min(rows[s], r0 + step)
            a = int(first[s])
            pos = torch.arange(keys[s] - rows[s] + r0, keys[s] - rows[s] + r1, device=DEVICE)[:, None]
            lo, hi = 0, keys[s] - rows[s] + r1
            j = torch.arange(lo, hi, device=DEVICE)[None]
            hidden = j > pos
            if case["op"] == "window":
                hidden |= (j <= pos - case["window"]) & (j >= case["sinks"])
            for h in range(hq):
                sc = st["q"][a + r0:a + r1, h].double() @ K[lo:hi, h // G].T / math.sqrt(hd)
                sc[hidden] = -torch.inf
                out[a + r0:a + r1, h] = torch.softmax(sc, -1) @ V[lo:hi, h // G]
    return out


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    rows, keys = _lens(case)
    hq, hkv, hd = case["hq"], case["hkv"], case["hd"]
    e = 2 if case["dtype"] == "bf16" else 4
    n = sum(rows)
    if case["op"] == "append":
        src = 2 if case["src"] == "bf16" else 4
        pos = len({p for k, r in zip(keys, rows) for p in range(k - r, k)})
        return dict(bytes=n * (hq + 2 * hkv) * hd * (src + e) + pos * hd * 4,
                    flops=n * (hq + hkv) * hd * (7 if case["norm"] else 3))
    seen = read = 0
    for r, k in zip(rows, keys):
        p = np.arange(k - r, k)
        if case["op"] == "window":
            w, t = case["window"], case["sinks"]
            low = np.maximum(p - w + 1, 0)                  # first key of the window
            seen += int((p + 1 - low + np.minimum(low, t)).sum())
            read += k - int(low[0]) + min(int(low[0]), t)
        else:
            seen += int((p + 1).sum())
            read += k - case["prefix"]
    read += case.get("prefix", 0)
    return dict(bytes=(2 * read * hkv + 2 * n * hq) * hd * e, flops=4 * seen * hq * hd)
