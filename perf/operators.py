"""Performance cases of the operators on a K/V cache: attention of new tokens
(one, a tree of drafted ones, a frame) over the cache, the accepted rows'
append, the accumulated attention weights of the cache's slots, and eviction
down to a budget of slots.

A cache holds [batch, kv_heads, capacity, d] keys and values of which the first
lengths[b] slots of batch entry b are in use, a score (accumulated attention
weight) and a token position for each slot.  Sizes are those of the package's
video workloads: frames of 30 x 52, 45 x 80 and 44 x 80 tokens, clips of 17,160
to 84,480 tokens, 16 heads, or 24 query heads on 8 K/V heads.

The plain forms compute in 32 bits by products, exponentials, comparisons and
indexing; exact() computes the same from the definitions in 64 bits, one batch
entry and K/V head at a time.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# One case.  kind: attend, accumulate, append, evict, step (append and evict in
# place).  len: slots in use of the first batch entry; with ragged = 1 later
# entries use fewer (down to half).  tokens: new tokens per entry; tree: 1 = the
# tokens form a tree, 0 = a chain.  rows: accepted tokens (accumulate, append;
# 0 = all).  budget, sink, recent: slots that are kept.
_DEFAULTS = dict(batch=1, heads=24, kv_heads=8, d=128, dtype="bf16", len=0, ragged=0, tokens=1,
                 tree=0, rows=0, budget=0, sink=0, recent=0)


def _case(**kw):
    return {**_DEFAULTS, **kw}


def listed():
    return [
        # one new token, a short cache: the first steps of a rollout, where
        # latency is all there is
        _case(name="attend_token_small", kind="attend", heads=8, kv_heads=2, len=1021),
        # a decoding step of four rollouts of different age over long caches
        _case(name="attend_token_long", kind="attend", batch=4, len=84480, ragged=1),
        # a tree of drafted tokens verified over a 720p clip's cache
        _case(name="attend_tree", kind="attend", batch=2, len=75600, ragged=1, tokens=63, tree=1),
        # a frame of 30 x 52 tokens in causal order over a clip at low resolution
        _case(name="attend_frame", kind="attend", len=17160, tokens=1560),
        # the fp32 path (validation runs), head dimension 64, a small tree
        _case(name="attend_tree_f32", kind="attend", batch=3, heads=12, kv_heads=4, d=64,
              dtype="f32", len=4335, ragged=1, tokens=29, tree=1),
        # the weights of an accepted path of a drafted tree
        _case(name="accumulate_path", kind="accumulate", batch=4, len=84480, ragged=1, tokens=63,
              rows=6),
        # the weights that a whole frame gives the cache and itself
        _case(name="accumulate_frame", kind="accumulate", len=18720, tokens=1560),
        # the fp32 path, head dimension 64
        _case(name="accumulate_f32", kind="accumulate", batch=3, heads=12, kv_heads=4, d=64,
              dtype="f32", len=4335, ragged=1, tokens=29, rows=7),
        # an accepted path enters a short cache
        _case(name="append_path", kind="append", batch=2, len=1021, ragged=1, tokens=29, rows=7),
        # two 44 x 80 frames enter the caches of a world model's two branches
        _case(name="append_frame", kind="append", batch=2, heads=16, kv_heads=16, len=42240,
              tokens=3520),
        # a clip's cache is cut down into a smaller one
        _case(name="evict_clip", kind="evict", batch=2, heads=16, kv_heads=16, len=17160, ragged=1,
              budget=4096, sink=64, recent=1560),
        # a rollout at its budget: an accepted path enters, as many slots leave
        _case(name="step_long", kind="step", batch=2, len=75600, budget=75600, tokens=63, rows=6,
              sink=64, recent=3600),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "accumulate", "accumulate", "append", "evict",
                       "step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 4, 8, 8, 16])
    heads = kv * rng.choice([1, 2, 3, 3, 4])
    batch = rng.choice([1, 1, 2, 3, 4])
    n = _log_uniform(rng, 200, 80000 if dtype == "bf16" else 9000)
    # at most the cache bytes of the largest listed case
    n = max(64, min(n, 2000000 // (kv * batch)))
    c = _case(kind=kind, batch=batch, heads=heads, kv_heads=kv, d=d, dtype=dtype, len=n,
              ragged=rng.choice([0, 1]))
    if kind in ("attend", "accumulate"):
        c["tree"] = rng.choice([0, 1])
        c["tokens"] = rng.choice([1, _log_uniform(rng, 2, 200), _log_uniform(rng, 2, 1500)])
        if c["tree"]:
            c["tokens"] = min(c["tokens"], 200)
        # at most the pairs of the frames
        most = 600000000 if dtype == "bf16" else 20000000
        c["tokens"] = max(1, min(c["tokens"], most // (batch * heads * n)))
        if kind == "accumulate":
            c["tree"] = 0
            c["tokens"] = min(c["tokens"], n)
            c["rows"] = rng.choice([0, max(1, c["tokens"] // 8)])
    elif kind == "append":
        c["ragged"] = 1
        c["tokens"] = max(2, min(_log_uniform(rng, 2, 3500), n // 2))
        c["rows"] = rng.choice([0, max(1, c["tokens"] // 6)])
    elif kind == "evict":
        c["budget"] = max(16, int(n * rng.uniform(0.1, 0.9)))
        c["recent"] = c["budget"] // 4
        c["sink"] = min(64, c["budget"] // 8)
    else:
        c["ragged"] = 0
        c["budget"] = n
        c["tokens"] = min(rng.choice([1, 17, 63]), n // 8)
        c["rows"] = rng.randint(1, min(7, c["tokens"]))
        c["recent"] = n // 8
        c["sink"] = min(64, n // 8)
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(case):
    n, b = case["len"], case["batch"]
    return [n - (i * n) // (2 * b) if case["ragged"] else n for i in range(b)]


def _counts(case):
    """Tokens (rows, where a list of accepted ones is given) of each entry."""
    n, b = case["rows"] or case["tokens"], case["batch"]
    return [max(1, n - (i * n) // (2 * b)) if case["ragged"] else n for i in range(b)]


def _capacity(case):
    grows = case["kind"] in ("append", "step")
    return case["len"] + (case["rows"] or case["tokens"] if grows else 0)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed % (1 << 62))
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    b, h, kv, d, t = (case[x] for x in ("batch", "heads", "kv_heads", "d", "tokens"))
    cap, kind = _capacity(case), case["kind"]

    def randn(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device=dev, dtype=torch.float32).mul_(scale).to(dt)

    def ints(x):
        return torch.tensor(np.asarray(x, np.int32), device=dev)

    # queries twice as long as keys: a row's weights spread over a part of the slots
    st = {"kind": kind, "k": randn(b, kv, cap, d), "v": randn(b, kv, cap, d),
          "lengths": ints(_lengths(case)), "counts": ints(_counts(case))}
    if kind in ("attend", "accumulate"):
        st["q"] = randn(b, h, t, d, scale=2.0)
    if kind in ("attend", "append", "step"):
        st["k_new"], st["v_new"] = randn(b, kv, t, d), randn(b, kv, t, d)
    if kind == "attend":
        st["out"] = torch.zeros(b, h, t, d, device=dev, dtype=dt)
        st["lse"] = torch.zeros(b, h, t, device=dev, dtype=torch.float32)
        st["parents"] = None
        if case["tree"]:
            # each token continues one of the few before it, or the root
            u = np.arange(t)
            st["parents"] = ints(np.maximum(u - 1 - rng.integers(0, 1 + np.minimum(u, 6), (b, t)), -1))
    else:
        # accumulated weights: few slots hold most of them.  Where rows add theirs, as
        # if about as many had done so before, so that neither part hides the other
        st["scores"] = torch.rand(b, kv, cap, generator=gen, device=dev).pow_(8.0).mul_(4.0)
        if kind == "accumulate":
            st["scores"].mul_(2.0 * (case["rows"] or t) * (h // kv) / case["len"])
        pos = torch.arange(cap, device=dev, dtype=torch.int32).expand(b, kv, cap)
        st["positions"] = pos.contiguous()
    if kind in ("accumulate", "append", "step"):
        st["rows"] = None
        if case["rows"]:
            st["rows"] = ints(np.stack([np.sort(rng.choice(t, case["rows"], replace=False))
                                        for _ in range(b)]))
    if kind == "accumulate":
        s, _ = _weights_logits(st)
        st["lse"] = torch.zeros(b, h, t, device=dev, dtype=torch.float32)
        idx = _rows(st).long()[:, None, :].expand(b, h, -1)
        st["lse"].scatter_(2, idx, torch.logsumexp(s, -1).reshape(b, h, -1))
        st["lse"].masked_fill_(st["lse"] == -math.inf, 0.0)
        del s
    if kind in ("append", "step"):
        # the tokens' positions follow the newest slot's
        st["new_positions"] = (ints(_lengths(case))[:, None] +
                               torch.arange(t, device=dev, dtype=torch.int32)[None]).contiguous()
        st["advance"] = case["rows"] or t
        st["new_lengths"] = torch.zeros(b, device=dev, dtype=torch.int32)
    if kind in ("evict", "step"):
        st.update({x: case[x] for x in ("budget", "sink", "recent")})
    if kind == "evict":
        # the smaller cache that the kept slots go to
        n = case["budget"]
        st["to"] = {"k": torch.zeros(b, kv, n, d, device=dev, dtype=dt),
                    "v": torch.zeros(b, kv, n, d, device=dev, dtype=dt),
                    "scores": torch.zeros(b, kv, n, device=dev),
                    "positions": torch.zeros(b, kv, n, device=dev, dtype=torch.int32),
                    "lengths": torch.zeros(b, device=dev, dtype=torch.int32)}
    if own:
        # the handles that a program keeps for its caches
        from paper_2608_18484_amd import sparsepr as S
        st["cache"] = S.KVCache(st["k"], st["v"], st["lengths"], scores=st.get("scores"),
                                positions=st.get("positions"))
        if kind == "evict":
            st["to_cache"] = S.KVCache(st["to"]["k"], st["to"]["v"], st["to"]["lengths"],
                                       scores=st["to"]["scores"], positions=st["to"]["positions"])
    torch.cuda.synchronize()
    return st


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _grouped(x, kv):
    """[B, H, T, d] as [B, kv, (H / kv) T, d] in 32 bits."""
    b, h, t, d = x.shape
    return x.float().reshape(b, kv, (h // kv) * t, d)


def _ancestors(parents):
    """[B, T, T]: entry (t, u) whether u is t or one of its ancestors."""
    b, t = parents.shape
    step = torch.eye(t, device=parents.device, dtype=torch.float64).repeat(b, 1, 1)
    u = torch.arange(t, device=parents.device)
    step += (parents[:, :, None] == u[None, None, :]).double()
    return torch.linalg.matrix_power(step, t) > 0


def _attend(st):
    q, k, v = st["q"], st["k"], st["v"]
    b, h, t, d = q.shape
    kv, cap = k.shape[1], k.shape[2]
    g = h // kv
    u = torch.arange(t, device=q.device)
    seen = torch.arange(cap, device=q.device)[None] < st["lengths"][:, None]
    if st["parents"] is None:
        mask = (u[:, None] >= u[None, :]).expand(b, t, t)
    else:
        mask = _ancestors(st["parents"])
    mask = torch.cat([seen[:, None, :].expand(b, t, cap), mask], 2)
    qf = _grouped(q, kv) / math.sqrt(d)
    s = torch.matmul(qf, torch.cat([k, st["k_new"]], 2).float().transpose(-1, -2).contiguous())
    s = s.view(b, kv, g, t, cap + t).masked_fill_(~mask[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = s.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, kv, g * t, cap + t), torch.cat([v, st["v_new"]], 2).float())
    o = o.view(b, h, t, d) / l.view(b, h, t, 1)
    lse = (m + l.log()).view(b, h, t)
    on = u[None, None, :] < st["counts"][:, None, None]
    st["out"].copy_(torch.where(on[..., None], o.to(q.dtype), st["out"]))
    st["lse"].copy_(torch.where(on, lse, st["lse"]))
    return {"out": st["out"], "lse": st["lse"]}


def _rows(st):
    """[B, C]: the accepted tokens, in their order."""
    if st["rows"] is not None:
        return st["rows"]
    b, t = (st["q"].shape[0], st["q"].shape[2]) if "q" in st else (st["k_new"].shape[0],
                                                                   st["k_new"].shape[2])
    return torch.arange(t, device=st["k"].device, dtype=torch.int32).expand(b, t)


def _weights_logits(st):
    """Logits [B, kv, g, C, capacity] of the accepted rows (-inf where a row
    does not see a slot) and their token indices."""
    q, k = st["q"], st["k"]
    b, h, t, d = q.shape
    kv, cap = k.shape[1], k.shape[2]
    rows = _rows(st).long()
    c = rows.shape[1]
    qr = q.gather(2, rows[:, None, :, None].expand(b, h, c, d))
    s = torch.matmul(_grouped(qr, kv) / math.sqrt(d), k.float().transpose(-1, -2).contiguous())
    i = torch.arange(c, device=q.device)[None]
    sees = (st["lengths"][:, None] - st["counts"][:, None] + i + 1).masked_fill(
        i >= st["counts"][:, None], 0)
    mask = torch.arange(cap, device=q.device)[None, None] < sees[..., None]
    return s.view(b, kv, h // kv, c, cap).masked_fill_(~mask[:, None, None], -math.inf), rows


def _accumulate(st):
    s, rows = _weights_logits(st)
    b, kv, g, c, _ = s.shape
    lse = st["lse"].gather(2, rows[:, None, :].expand(b, kv * g, c))
    st["scores"] += s.sub_(lse.view(b, kv, g, c, 1)).exp_().sum((2, 3))
    return {"scores": st["scores"]}


def _append(st, lengths_out):
    rows = _rows(st).long()
    b, c = rows.shape
    i = torch.arange(c, device=rows.device)[None]
    bi, ri = torch.nonzero(i < st["counts"][:, None], as_tuple=True)
    slot = st["lengths"].long()[bi] + ri
    tok = rows[bi, ri]
    st["k"][bi, :, slot] = st["k_new"][bi, :, tok]
    st["v"][bi, :, slot] = st["v_new"][bi, :, tok]
    st["scores"][bi, :, slot] = 0.0
    st["positions"][bi, :, slot] = st["new_positions"][bi, tok][:, None].expand(-1, st["k"].shape[1])
    lengths_out.copy_(st["lengths"] + st["counts"])


def _sources(st):
    """[B, kv, budget]: the slot that goes to each kept slot (itself where it
    stays), and the new lengths."""
    sc, pos, n = st["scores"], st["positions"], st["budget"]
    cap = sc.shape[2]
    slot = torch.arange(cap, device=sc.device)
    used = slot[None] < st["lengths"][:, None]
    used = used[:, None, :].expand_as(sc)
    newest = pos.masked_fill(~used, -1).amax(2, keepdim=True)
    safe = (pos < st["sink"]) | (pos > newest - st["recent"])
    rank = torch.where(safe, torch.full_like(sc, math.inf), sc).masked_fill(~used, -math.inf)
    order = rank.argsort(dim=2, descending=True, stable=True)[:, :, :n]
    keep = torch.zeros_like(used).scatter(2, order, True) & used
    late = keep & (slot >= n)
    movers = (~late).to(torch.int8).argsort(dim=2, stable=True)[:, :, :n]
    hole = ~keep[:, :, :n]
    nth = hole.cumsum(2) - 1
    fill = hole & (nth < late.sum(2, keepdim=True))
    here = slot[:n].expand(*fill.shape)
    src = torch.where(fill, movers.gather(2, nth.clamp(min=0)), here)
    return src, st["lengths"].clamp(max=n)


def _evict(st, to):
    src, lengths = _sources(st)
    b, kv, n = src.shape
    valid = torch.arange(n, device=src.device)[None, None] < lengths[:, None, None]
    for x in ("k", "v", "scores", "positions"):
        idx = src if x in ("scores", "positions") else src[..., None].expand(*src.shape, st[x].shape[3])
        ok = valid if x in ("scores", "positions") else valid[..., None]
        to[x][:, :, :n] = torch.where(ok, st[x].gather(2, idx), to[x][:, :, :n])
    to["lengths"].copy_(lengths)
    return {x: to[x] for x in ("k", "v", "scores", "positions", "lengths")}


def run(state):
    st, kind = state, state["kind"]
    if kind == "step":
        # positions go on from step to step
        st["new_positions"] += st["advance"]
    if not own:
        if kind == "attend":
            return _attend(st)
        if kind == "accumulate":
            return _accumulate(st)
        if kind == "append":
            _append(st, st["new_lengths"])
            return {**{x: st[x] for x in ("k", "v", "scores", "positions")},
                    "lengths": st["new_lengths"]}
        if kind == "evict":
            return _evict(st, st["to"])
        _append(st, st["lengths"])
        return _evict(st, st)
    cache = st["cache"]
    if kind == "attend":
        cache.attend(st["q"], st["k_new"], st["v_new"], parents=st["parents"],
                     counts=st["counts"], out=st["out"], lse=st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "accumulate":
        cache.accumulate(st["q"], st["lse"], rows=st["rows"], counts=st["counts"])
        return {"scores": st["scores"]}
    if kind == "append":
        cache.append(st["k_new"], st["v_new"], positions=st["new_positions"], rows=st["rows"],
                     counts=st["counts"], lengths_out=st["new_lengths"])
        return {**{x: st[x] for x in ("k", "v", "scores", "positions")},
                "lengths": st["new_lengths"]}
    if kind == "evict":
        cache.evict(st["budget"], n_sink=st["sink"], n_recent=st["recent"], out=st["to_cache"])
        return {x: st["to"][x] for x in ("k", "v", "scores", "positions", "lengths")}
    cache.append(st["k_new"], st["v_new"], positions=st["new_positions"], rows=st["rows"],
                 counts=st["counts"])
    cache.evict(st["budget"], n_sink=st["sink"], n_recent=st["recent"])
    return {x: st[x] for x in ("k", "v", "scores", "positions", "lengths")}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Slots in use, new rows and outputs moved once; 4 d flops per visible
    pair of the attention, 2 d per pair of the weights."""
    size = 2 if case["dtype"] == "bf16" else 4
    h, kv, d, t, kind = (case[x] for x in ("heads", "kv_heads", "d", "tokens", "kind"))
    row, ls, cs = kv * d * size, _lengths(case), _counts(case)
    byts = flops = 0
    for l, c in zip(ls, cs):
        if kind == "attend":
            byts += 2 * row * (l + c) + 2 * h * d * size * c + 4 * h * c
            # of a tree's tokens a row sees a few
            flops += 4 * d * h * c * (l + ((c + 1) / 2 if not case["tree"] else math.log2(c + 1)))
        elif kind == "accumulate":
            byts += row * l + 8 * kv * l + h * d * size * c + 4 * h * c
            flops += 2 * d * h * c * (l - (c - 1) / 2)
        if kind in ("append", "step"):
            byts += 4 * row * c + 12 * kv * c
        if kind == "evict":
            n = min(l, case["budget"])
            byts += 8 * kv * l + 4 * row * n + 8 * kv * n
        if kind == "step":
            byts += 8 * kv * (l + c) + 4 * row * c + 16 * kv * c
    return {"bytes": int(byts), "flops": int(flops)}


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _exact_attend(st, case, ls, cs):
    q, kv = st["q"], case["kv_heads"]
    b, h, t, d = q.shape
    g = h // kv
    out, lse = st["out"].double(), st["lse"].double()
    par = None if st["parents"] is None else st["parents"].cpu().numpy()
    for i in range(b):
        n, c = ls[i], cs[i]
        see = torch.zeros(c, c, dtype=torch.bool)
        for u in range(c):
            if par is None:
                see[u, :u + 1] = True
            else:
                w = u
                while w >= 0:
                    see[u, w] = True
                    w = int(par[i, w])
        see = see.to(q.device)
        for j in range(kv):
            kc, vc = st["k"][i, j, :n].double(), st["v"][i, j, :n].double()
            kn, vn = st["k_new"][i, j, :c].double(), st["v_new"][i, j, :c].double()
            for x in range(j * g, (j + 1) * g):
                qx = q[i, x, :c].double() / math.sqrt(d)
                a, e = qx @ kc.T, (qx @ kn.T).masked_fill(~see, -math.inf)
                z = torch.logaddexp(torch.logsumexp(a, 1), torch.logsumexp(e, 1)) if n else \
                    torch.logsumexp(e, 1)
                out[i, x, :c] = torch.exp(a - z[:, None]) @ vc + torch.exp(e - z[:, None]) @ vn
                lse[i, x, :c] = z
    return {"out": out, "lse": lse}


def _exact_accumulate(st, case, ls, cs):
    q, kv = st["q"], case["kv_heads"]
    b, h, t, d = q.shape
    g = h // kv
    sc = st["scores"].double()
    for i in range(b):
        n, c = ls[i], cs[i]
        tok = torch.arange(c) if st["rows"] is None else st["rows"][i, :c].long().cpu()
        tok = tok.to(q.device)
        last = n - c + torch.arange(c, device=q.device)  # the last slot that each row sees
        for x in range(h):
            j = x // g
            a = (q[i, x][tok].double() @ st["k"][i, j, :n].double().T) / math.sqrt(d)
            a -= st["lse"][i, x][tok].double()[:, None]
            a.masked_fill_(torch.arange(n, device=q.device)[None] > last[:, None], -math.inf)
            sc[i, j, :n] += a.exp_().sum(0)
    return {"scores": sc}


def _exact_append(x, st, case, ls, cs, positions):
    for i in range(case["batch"]):
        n, c = ls[i], cs[i]
        tok = np.arange(c) if st["rows"] is None else st["rows"][i, :c].cpu().numpy()
        for r, u in enumerate(tok):
            x["k"][i, :, n + r] = st["k_new"][i, :, u].double()
            x["v"][i, :, n + r] = st["v_new"][i, :, u].double()
            x["scores"][i, :, n + r] = 0.0
            x["positions"][i, :, n + r] = positions[i, u]
        x["lengths"][i] = n + c


def _exact_evict(x, to, case):
    n = case["budget"]
    for i in range(case["batch"]):
        length = int(x["lengths"][i])
        to["lengths"][i] = min(length, n)
        for j in range(case["kv_heads"]):
            score = x["scores"][i, j, :length].cpu().numpy()
            pos = x["positions"][i, j, :length].cpu().numpy().astype(np.int64)
            safe = (pos < case["sink"]) | (pos >= pos.max() - case["recent"] + 1)
            order = np.lexsort((np.arange(length), -score, ~safe))
            keep = np.sort(order[:n])
            stay, late = keep[keep < n], keep[keep >= n]
            free = np.setdiff1d(np.arange(min(n, length)), stay)
            src = torch.from_numpy(np.concatenate([stay, late]))
            dst = torch.from_numpy(np.concatenate([stay, free]))
            dev = x["k"].device
            for y in ("k", "v", "scores", "positions"):
                to[y][i, j][dst.to(dev)] = x[y][i, j][src.to(dev)]


def exact(case, seed):
    st = prepare(case, seed)
    kind, ls, cs = case["kind"], _lengths(case), _counts(case)
    if kind == "attend":
        return _exact_attend(st, case, ls, cs)
    if kind == "accumulate":
        return _exact_accumulate(st, case, ls, cs)
    x = {y: st[y].double() for y in ("k", "v", "scores")}
    x.update({y: st[y].clone() for y in ("positions", "lengths")})
    if kind == "append":
        _exact_append(x, st, case, ls, cs, st["new_positions"])
        return x
    if kind == "evict":
        to = {y: st["to"][y].double() for y in ("k", "v", "scores")}
        to.update({y: st["to"][y].clone() for y in ("positions", "lengths")})
        _exact_evict(x, to, case)
        return to
    _exact_append(x, st, case, ls, cs, st["new_positions"] + st["advance"])
    to = {y: x[y].clone() for y in x}
    _exact_evict(x, to, case)
    return to
