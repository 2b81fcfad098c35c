"""Performance cases of the calls around a larger model's tokens: log-probabilities of given tokens
with entropies and alternatives, their gradient, the paged cache's append with the rotation of
positions, and attention of drafted tokens (a tree or a path) over that cache: what they compute,
on which inputs, what one pass cannot do without, and the same results in float64.

A case is a dict of plain values:
  op       score    log-probability of a given token of every row, the row's entropy, and its K
                    most likely tokens with theirs
           grad     the same without alternatives, with the gradient of
                    sum(weights * logp + entropy_weights * entropy)
           append   keys and values of new tokens into a paged cache, keys and queries rotated
           attend   drafted tokens' queries over the cache
  dtype    float32, bfloat16, float16 (append, attend: the last two)
  B, N     sequences, and tokens of each (append: new ones, attend: drafted ones)
  lengths  full     every sequence has N tokens
           half     uniform in [N / 2, N]
           any      uniform in [0, N], not 0 for the first
score, grad:
  V, K     vocabulary; alternatives
  pitch    a row's elements in memory (>= V)
  T        temperature
  entropy  grad: the entropy has a weight too
append, attend:
  Hq, Hk, D  heads of queries, of keys and values (a divisor of Hq), elements of a head
  page     tokens of a page
  past     most tokens in the cache before these; every sequence has between spread * past and past
  R        append: rotated elements of a head; pairs: halves (i, i + R / 2) or neighbours (2i, 2i + 1)
  tree     attend: a tree of drafts, otherwise a path
"""
import math

import numpy as np
import torch

DEV = "cuda:0"
own = False

MAX_ELEMENTS = 4 * 2048 * 131072          # logits of the largest listed case
MAX_SORTED = 4 * 1024 * 131072            # and of the largest listed `score`
MAX_PLAIN = 6 << 30                       # bytes that a drawn attention's plain form holds
MAX_CACHE = 300 << 20                     # bytes of keys and values that it reads
MAX_FLOPS = 8e10
CHUNK = 1 << 26                           # elements that exact() holds at once


def _rows(name, op, B, N, V, K, dtype, lengths="full", pitch=0, T=1.0, entropy=False):
    return dict(name=name, op=op, B=B, N=N, V=V, K=K, dtype=dtype, lengths=lengths,
                pitch=max(V, pitch), T=T, entropy=entropy)


def _append(name, B, N, Hq, Hk, D, dtype, page, past, R, pairs="halves", lengths="full", spread=0.5):
    return dict(name=name, op="append", B=B, N=N, Hq=Hq, Hk=Hk, D=D, dtype=dtype, page=page,
                past=past, spread=spread, lengths=lengths, R=R, pairs=pairs)


def _attend(name, B, N, Hq, Hk, D, dtype, page, past, tree=True, lengths="full", spread=0.5):
    return dict(name=name, op="attend", B=B, N=N, Hq=Hq, Hk=Hk, D=D, dtype=dtype, page=page,
                past=past, spread=spread, lengths=lengths, tree=tree)


def listed():
    return [
        # a small tagger's batch: the log-probabilities of its gold labels, five best beside them
        _rows("score_labels", "score", 32, 25, 20, 5, "float32", "half"),
        # answers of a serving batch scored over a medium vocabulary, eight alternatives a token
        _rows("score_mid", "score", 8, 500, 32000, 8, "bfloat16", "half", T=0.7),
        # long documents scored over a large vocabulary
        _rows("score_large", "score", 4, 1024, 131072, 20, "bfloat16"),
        # a tagger's training step on given labels
        _rows("grad_labels", "grad", 32, 25, 20, 0, "float32", "half"),
        # a policy's step with its entropy bonus, an odd vocabulary in rows of an aligned pitch
        _rows("grad_policy", "grad", 7, 301, 50001, 0, "bfloat16", "half", pitch=50048, T=1.5,
              entropy=True),
        # a likelihood step of long sequences over a large vocabulary
        _rows("grad_large", "grad", 4, 2048, 131072, 0, "bfloat16"),
        # one token of one user: latency
        _append("append_one", 1, 1, 32, 8, 128, "bfloat16", 16, 4000, 128),
        # prompts of unequal lengths taken into the cache
        _append("append_prompts", 8, 2048, 32, 8, 128, "bfloat16", 64, 1000, 128, lengths="half",
                spread=0.0),
        # one user's tree of sixteen drafts: latency
        _attend("attend_one", 1, 16, 32, 8, 128, "bfloat16", 16, 2000),
        # a serving batch, a path of up to five drafts each, contexts of unequal lengths
        _attend("attend_batch", 64, 5, 32, 8, 128, "bfloat16", 16, 8000, tree=False, lengths="any",
                spread=0.1),
        # wide trees over medium contexts: bound by the products
        _attend("attend_wide", 8, 64, 64, 8, 128, "bfloat16", 64, 4500, spread=0.9),
        # one long document, few rows, an odd number of query heads a key head, an odd page
        _attend("attend_long", 1, 7, 28, 4, 64, "float16", 48, 131072, spread=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["score", "grad", "append", "attend", "attend"])
    if op in ("score", "grad"):
        while True:
            V, B, N = _log_int(rng, 16, 262144), _log_int(rng, 1, 32), _log_int(rng, 1, 4096)
            if B * N * V <= (MAX_SORTED if op == "score" else MAX_ELEMENTS // 2):
                break
        c = _rows("", op, B, N, V, 0 if op == "grad" else rng.choice([0, _log_int(rng, 1, min(V, 64))]),
                  rng.choice(["float32", "bfloat16", "bfloat16", "float16"]),
                  lengths=rng.choice(["full", "half"]),
                  pitch=V if rng.random() < 0.5 else (V + 63) // 64 * 64,
                  T=rng.choice([1.0, 1.0, 0.7, 2.0]), entropy=op == "grad" and rng.random() < 0.5)
        del c["name"]
        return c
    dtype = rng.choice(["bfloat16", "bfloat16", "float16"])
    Hk = rng.choice([1, 2, 4, 8])
    Hq = Hk * rng.choice([1, 2, 4, 7, 8])
    D, page = rng.choice([64, 80, 128, 128, 256]), rng.choice([1, 16, 16, 48, 64, 128])
    lengths, spread = rng.choice(["full", "half", "any"]), rng.choice([0.0, 0.5, 1.0])
    while True:
        B = _log_int(rng, 1, 64)
        if op == "append":
            N, past = _log_int(rng, 1, 4096), _log_int(rng, 1, 8192)
            if B * N * (Hq + 2 * Hk) * D <= 8 * 2048 * 48 * 128 and \
                    B * (N + past) * Hk * D <= 1 << 28:
                break
        else:
            N, past = _log_int(rng, 1, 128), _log_int(rng, 1, 131072)
            keys = B * (past + N) * Hk
            if keys * (4 * D + 3 * N * (Hq // Hk)) * 4 <= MAX_PLAIN and \
                    keys * 4 * D <= MAX_CACHE and 4 * keys * N * (Hq // Hk) * D <= MAX_FLOPS:
                break
    if op == "append":
        c = _append("", B, N, Hq, Hk, D, dtype, page, past, rng.choice([D, D // 32 * 16]),
                    rng.choice(["halves", "neighbours"]), lengths, spread)
    else:
        c = _attend("", B, N, Hq, Hk, D, dtype, page, past, rng.random() < 0.7, lengths, spread)
    del c["name"]
    return c


# ---- inputs ----

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _ints(host):
    return torch.from_numpy(host.astype(np.int32)).to(DEV)


def _lengths(case, rng):
    B, N = case["B"], case["N"]
    lo = {"full": N, "half": max(1, N // 2), "any": 0}[case["lengths"]]
    n = rng.integers(lo, N, endpoint=True, size=B)
    n[0] = max(n[0], 1)
    return _ints(n)


def prepare(case, seed):
    rng, g = np.random.default_rng(seed), _generator(seed)
    st = {"case": case, "lengths": _lengths(case, rng)}
    if case["op"] in ("score", "grad"):
        return _prepare_rows(case, g, st)
    return _prepare_cache(case, rng, g, st)


def _prepare_rows(case, g, st):
    # a language model's rows: most of the vocabulary in a broad bulk, a few tokens far above
    B, N, V = case["B"], case["N"], case["V"]
    k = min(V, 16)
    step = V // k
    at = torch.randint(0, step, (B, N, k), generator=g, device=DEV)
    at += torch.arange(k, device=DEV) * step
    peaks = 13.0 - 2.0 * torch.log1p(torch.arange(k, device=DEV)) + torch.randn(
        (B, N, k), generator=g, device=DEV)
    x = torch.randn((B, N, case["pitch"]), generator=g, device=DEV,
                    dtype=getattr(torch, case["dtype"]))
    x.mul_(2.0)
    x.scatter_(2, at, peaks.to(x.dtype))
    # the given tokens: mostly likely ones, some from the bulk
    z = at.gather(2, torch.randint(0, k, (B, N, 1), generator=g, device=DEV))[..., 0]
    any_z = torch.randint(0, V, (B, N), generator=g, device=DEV)
    rare = torch.rand((B, N), generator=g, device=DEV) < 0.1
    st["logits"], st["tokens"] = x[..., :V], torch.where(rare, any_z, z).to(torch.int32)
    if case["op"] == "grad":
        st["weights"] = torch.randn((B, N), generator=g, device=DEV)
        st["entropy_weights"] = None
        if case["entropy"]:
            st["entropy_weights"] = 0.01 + 0.1 * torch.rand((B, N), generator=g, device=DEV)
    return st


def _prepare_cache(case, rng, g, st):
    B, N, Hq, Hk, D, S = (case[k] for k in ("B", "N", "Hq", "Hk", "D", "page"))
    dtype = getattr(torch, case["dtype"])
    starts = rng.integers(int(case["spread"] * case["past"]), case["past"], endpoint=True, size=B)
    each = (starts + N + S - 1) // S
    wide = int((case["past"] + N + S - 1) // S)
    pool = B * wide + 3
    ids = rng.permutation(pool)[:int(each.sum())]   # a cache in use: pages lie anywhere in it
    pages = np.full((B, wide), -1, dtype=np.int64)
    pages[np.arange(wide)[None] < each[:, None]] = ids
    st["starts"], st["pages"] = _ints(starts), _ints(pages)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dtype)

    st["k_cache"], st["v_cache"] = normal(pool, S, Hk, D), normal(pool, S, Hk, D)
    if case["op"] == "append":
        # what one product for queries, keys and values leaves: views of its rows
        qkv = normal(B, N, Hq + 2 * Hk, D)
        st["q"], st["k"], st["v"] = qkv.split([Hq, Hk, Hk], 2)
        R = case["R"]
        st["freqs"] = (10000.0 ** (-torch.arange(0, R, 2, device=DEV).double() / R)).float()
        return st
    st["q"] = normal(B, N, Hq, D).mul_(1.5)
    st["parents"] = None
    if case["tree"]:
        # most drafts continue one of the last few, some begin a branch of their own
        back = rng.integers(1, 8, endpoint=True, size=(B, N))
        st["parents"] = _ints(np.maximum(np.arange(N)[None] - back, -1))
    return st


# ---- one pass ----

def run(state):
    return (_calls if own else _plain)(state)


def _calls(st):
    from paper_2002_00876_amd import binding

    case, n = st["case"], st["lengths"]
    op = case["op"]
    if op == "score":
        return binding.score(st["logits"], st["tokens"], case["K"], n, temperature=case["T"])
    if op == "grad":
        return binding.score_grad(st["logits"], st["tokens"], n, weights=st["weights"],
                                  entropy_weights=st["entropy_weights"], temperature=case["T"])
    if op == "append":
        q = binding.cache_append(st["k"], st["v"], st["k_cache"], st["v_cache"], st["pages"],
                                 st["starts"], n, q=st["q"], freqs=st["freqs"],
                                 neighbours=case["pairs"] == "neighbours")
        return q, st["k_cache"], st["v_cache"]
    return binding.tree_attention(st["q"], st["k_cache"], st["v_cache"], st["pages"], st["starts"],
                                  st["parents"], n)


def _on(st):
    return torch.arange(st["case"]["N"], device=DEV)[None] < st["lengths"][:, None]


def _plain(st):
    op = st["case"]["op"]
    if op == "append":
        return _plain_append(st)
    if op == "attend":
        return _plain_attend(st)
    return _plain_rows(st)


def _plain_rows(st):
    case, on = st["case"], _on(st)
    x = st["logits"].float()
    a = x / case["T"]
    m = a.amax(2, keepdim=True)
    d = a - m
    e = d.exp()
    s = e.sum(2)
    ls = s.log()
    # log s and the mean distance to the maximum, neither of them negative
    entropy = torch.where(on, ls - (d * e).sum(2) / s, 0.0)
    z = st["tokens"].long()[..., None]
    logp = torch.where(on, d.gather(2, z)[..., 0] - ls, 0.0)
    if case["op"] == "score":
        K = case["K"]
        # equal logits: the lowest index first
        v, i = x.sort(dim=2, descending=True, stable=True)
        top = v[..., :K] / case["T"] - (m[..., 0] + ls)[..., None]
        return (logp, entropy, i[..., :K].to(torch.int32).masked_fill(~on[..., None], -1),
                top.masked_fill(~on[..., None], -math.inf))
    w = torch.where(on, st["weights"], 0.0)[..., None] / case["T"]
    p = e / s[..., None]
    grad = p * -w
    grad.scatter_add_(2, z, w)
    if st["entropy_weights"] is not None:
        u = torch.where(on, st["entropy_weights"], 0.0)[..., None] / case["T"]
        grad -= u * p * (d - ls[..., None] + entropy[..., None])
    return logp, entropy, grad.to(st["logits"].dtype)


def _rotated(x, st):
    """The first R elements of every head turned by the position's angles, formed in 64 bits."""
    case, h = st["case"], st["case"]["R"] // 2
    at = st["starts"][:, None] + torch.arange(case["N"], device=DEV)[None]
    angle = at.double()[..., None, None] * st["freqs"].double()
    c, s = angle.cos().float(), angle.sin().float()
    x = x.float()
    y = x.clone()
    one, two = ((slice(0, h), slice(h, 2 * h)) if case["pairs"] == "halves" else
                (slice(0, 2 * h, 2), slice(1, 2 * h, 2)))
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    return y


def _plain_append(st):
    case, on, S = st["case"], _on(st), st["case"]["page"]
    slot = st["starts"].long()[:, None] + torch.arange(case["N"], device=DEV)[None]
    page = st["pages"].long().gather(1, slot // S)
    at = (page * S + slot % S)[on]
    kc, vc = st["k_cache"], st["v_cache"]
    kc.view(-1, *kc.shape[2:])[at] = _rotated(st["k"], st)[on].to(kc.dtype)
    vc.view(-1, *vc.shape[2:])[at] = st["v"][on]
    q = torch.where(on[..., None, None], _rotated(st["q"], st), 0.0)
    return q.to(st["q"].dtype), kc, vc


def _ancestors(parents, B, N):
    """[B, N, N]: whether the second is the first or one that it follows."""
    at = torch.arange(N, device=DEV)
    if parents is None:
        return (at[None, :] <= at[:, None])[None].expand(B, N, N)
    reach = ((parents[..., None] == at) | (at[:, None] == at)).float()
    for _ in range(N.bit_length()):               # paths of 1, 2, 4, ... steps
        reach = (torch.bmm(reach, reach) > 0).float()
    return reach > 0


def _plain_attend(st):
    case, q, S = st["case"], st["q"], st["case"]["page"]
    B, N, Hq, D = q.shape
    Hk = case["Hk"]
    G, L = Hq // Hk, case["past"] + N
    slot = torch.arange(L, device=DEV)
    page = st["pages"].long()[:, slot // S].clamp(min=0)
    k = st["k_cache"][page, slot % S].permute(0, 2, 3, 1).contiguous().float()
    v = st["v_cache"][page, slot % S].permute(0, 2, 1, 3).contiguous().float()
    qg = q.float().view(B, N, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, N * G, D)
    s = torch.matmul(qg, k) * D ** -0.5
    since = slot[None] - st["starts"][:, None]
    seen = _ancestors(st["parents"], B, N).gather(
        2, since.clamp(0, N - 1)[:, None].expand(B, N, L).long())
    seen = torch.where((since < 0)[:, None], True, seen & (since < N)[:, None])
    s = s.view(B, Hk, N, G, L).masked_fill(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = (s - m).exp()
    l = p.sum(-1, keepdim=True)
    out = torch.matmul((p / l).view(B, Hk, N * G, L), v).view(B, Hk, N, G, D)
    out = out.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, D)
    lse = (m + l.log()).view(B, Hk, N, G).permute(0, 2, 1, 3).reshape(B, N, Hq)
    on = _on(st)[..., None]
    return torch.where(on[..., None], out, 0.0).to(q.dtype), lse.masked_fill(~on, -math.inf)


# ---- what a pass cannot do without ----

def work(case):
    B, N = case["B"], case["N"]
    size = 4 if case["dtype"] == "float32" else 2
    rows = B * N * {"full": 1.0, "half": 0.75, "any": 0.5}[case["lengths"]]
    if case["op"] in ("score", "grad"):
        V, K = case["V"], case["K"]
        logits = rows * V
        if case["op"] == "score":
            return {"bytes": int(logits * size + 4 * rows + B * N * (8 + 8 * K)),
                    "flops": int(5 * logits)}
        weights = 8 if case["entropy"] else 4
        # the gradient is written for padding too
        return {"bytes": int((logits + B * N * V) * size + (4 + weights) * rows + 8 * B * N),
                "flops": int((10 if case["entropy"] else 7) * logits)}
    Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
    if case["op"] == "append":
        # queries, keys and values read and written; queries are written for padding too
        moved = rows * (Hq + 4 * Hk) * D + B * N * Hq * D
        return {"bytes": int(moved * size + rows * 4 / case["page"]),
                "flops": int(3 * rows * (Hq + Hk) * case["R"])}
    keys = B * case["past"] * (1 + case["spread"]) / 2 + rows
    return {"bytes": int(2 * keys * Hk * D * size + (rows + B * N) * Hq * D * size +
                         4 * B * N * Hq + 4 * keys / case["page"] + (4 * rows if case["tree"] else 0)),
            "flops": int(4 * (keys / B) * rows * Hq * D)}


# ---- the same results in float64 ----

def exact(case, seed):
    st = prepare(case, seed)
    n = st["lengths"].tolist()
    if case["op"] in ("score", "grad"):
        return _exact_rows(st, n)
    return _exact_append(st, n) if case["op"] == "append" else _exact_attend(st, n)


def _exact_rows(st, n):
    case = st["case"]
    B, N, V, K, T = case["B"], case["N"], case["V"], case["K"], case["T"]
    f64 = dict(dtype=torch.float64, device=DEV)
    logp, entropy = torch.zeros((B, N), **f64), torch.zeros((B, N), **f64)
    top = torch.full((B, N, K), -math.inf, **f64)
    grad = torch.zeros((B, N, V), **f64) if case["op"] == "grad" else None
    step = max(1, CHUNK // V)
    for b in range(B):
        for i in range(0, n[b], step):
            j = min(n[b], i + step)
            lp = torch.log_softmax(st["logits"][b, i:j].double() / T, 1)
            z = st["tokens"][b, i:j].long()
            p = lp.exp()
            h = -(p * lp).sum(1)
            at = torch.arange(j - i, device=DEV)
            logp[b, i:j], entropy[b, i:j] = lp[at, z], h
            if grad is None:
                top[b, i:j] = lp.topk(K, 1).values
                continue
            w = st["weights"][b, i:j].double()
            d = -w[:, None] * p
            d[at, z] += w
            if st["entropy_weights"] is not None:
                d -= st["entropy_weights"][b, i:j].double()[:, None] * p * (lp + h[:, None])
            grad[b, i:j] = d / T
    return (logp, entropy, None, top) if grad is None else (logp, entropy, grad)


def _exact_turn(x, at, st):
    """Rows x [n, H, D] of positions at [n]: pairs as complex numbers, multiplied by e^(i angle)."""
    case, R = st["case"], st["case"]["R"]
    x = x.double()
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       at.double()[:, None] * st["freqs"].double())[:, None]
    if case["pairs"] == "halves":
        z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * turn
        first = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous()) * turn
        first = torch.view_as_real(z).reshape(*x.shape[:-1], R)
    return torch.cat([first, x[..., R:]], -1)


def _exact_append(st, n):
    S = st["case"]["page"]
    q = torch.zeros_like(st["q"], dtype=torch.float64)
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    for b in range(st["case"]["B"]):
        at = st["starts"][b].long() + torch.arange(n[b], device=DEV)
        page = st["pages"][b].long()[at // S]
        kc[page, at % S] = _exact_turn(st["k"][b, :n[b]], at, st)
        vc[page, at % S] = st["v"][b, :n[b]].double()
        q[b, :n[b]] = _exact_turn(st["q"][b, :n[b]], at, st)
    return q, kc, vc


def _exact_attend(st, n):
    case, S = st["case"], st["case"]["page"]
    B, N, Hq, Hk, D = (case[k] for k in ("B", "N", "Hq", "Hk", "D"))
    G = Hq // Hk
    out = torch.zeros((B, N, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, N, Hq), -math.inf, dtype=torch.float64, device=DEV)
    starts = st["starts"].tolist()
    parents = None if st["parents"] is None else st["parents"].tolist()
    for b in range(B):
        m, L = n[b], starts[b] + n[b]
        if m == 0:
            continue
        hide = np.zeros((m, L), dtype=bool)
        hide[:, starts[b]:] = True
        for i in range(m):
            j = i
            while j >= 0:
                hide[i, starts[b] + j] = False
                j = j - 1 if parents is None else parents[b][j]
        hide = torch.from_numpy(hide).to(DEV)[:, None]
        slot = torch.arange(L, device=DEV)
        page = st["pages"][b].long()[slot // S]
        for h in range(Hk):
            k, v = (st[x][page, slot % S, h].double() for x in ("k_cache", "v_cache"))
            q = st["q"][b, :m, h * G:(h + 1) * G].double()
            s = (q.reshape(m * G, D) @ k.t()).view(m, G, L) / math.sqrt(D)
            s = s.masked_fill(hide, -math.inf)
            lse[b, :m, h * G:(h + 1) * G] = torch.logsumexp(s, 2)
            out[b, :m, h * G:(h + 1) * G] = (torch.softmax(s, 2).view(m * G, L) @ v).view(m, G, D)
    return out, lse
