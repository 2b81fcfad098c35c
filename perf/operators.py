"""Performance cases of the calls on rows of token logits: what they compute, on which inputs,
what one pass cannot do without, and the same results in float64.

A case is a dict of plain values:
  op       top      the K largest logits of every row and its log-sum-exp
           distill  the divergence of a student's rows from a teacher's top logits
           grad     the same with its gradient
           verify   drafted tokens against the target's probabilities
  B, N, V  sequences, tokens (verify: drafted tokens), vocabulary
  K        logits kept of a row (verify: 0)
  dtype    of the logits: float32, bfloat16, float16
  lengths  full     every sequence has N tokens
           half     uniform in [N / 2, N]
           any      uniform in [0, N] (verify)
  pitch    a row's elements in memory (>= V)
  rest     distill, grad: the teacher's log-sum-exp is given, and what its top logits leave is one
           class; otherwise they are normalised among themselves
           verify: the drafts' log-sum-exps are given
  ragged   distill, grad: a row has between 1 and K teacher logits
  T        temperature
"""
import math

import numpy as np
import torch

DEV = "cuda:0"
own = False

MAX_ELEMENTS = 8192 * 131072              # logits of the largest listed case
MAX_SORTED = 2048 * 131072                # and of the largest listed `top`
MIN_REST = 2.0 ** -20                     # a teacher's rest below this is the rounding of its parts
CHUNK = 1 << 26                           # elements that exact() holds at once


def _case(name, op, B, N, V, K, dtype, lengths="full", pitch=0, rest=False, ragged=False, T=1.0):
    return dict(name=name, op=op, B=B, N=N, V=V, K=K, dtype=dtype, lengths=lengths,
                pitch=max(V, pitch), rest=rest, ragged=ragged, T=T)


def listed():
    return [
        # label scores of one batch of a small tagger: its five best labels a token
        _case("top_labels", "top", 32, 25, 20, 5, "float32", "half"),
        # a teacher's logits over a medium vocabulary, taken while it trains a student
        _case("top_mid", "top", 8, 512, 32000, 32, "bfloat16", "half"),
        # a teacher's pass over long documents, its top logits written to a data set
        _case("top_large", "top", 4, 512, 131072, 128, "bfloat16"),
        # a tagger's training step from a larger tagger's posteriors
        _case("grad_labels", "grad", 32, 25, 20, 4, "float32", "half", rest=True),
        # a byte-level student held out: the loss alone
        _case("distill_bytes", "distill", 16, 1024, 256, 16, "float16", T=2.0),
        # held-out loss in 32 bits, unequal numbers of teacher logits
        _case("distill_mid", "distill", 8, 512, 32000, 64, "float32", "half", ragged=True),
        # one short sequence over the largest vocabulary: few rows, long ones
        _case("grad_few", "grad", 1, 9, 262144, 50, "float32", rest=True),
        # an odd vocabulary in rows of an aligned pitch
        _case("grad_odd", "grad", 7, 301, 50001, 100, "bfloat16", "half", pitch=50048, rest=True,
              ragged=True, T=1.5),
        # a training step of long sequences over a large vocabulary
        _case("grad_large", "grad", 4, 2048, 131072, 64, "bfloat16"),
        # a chain over bytes as the drafter (its rows are normalised), a few sequences
        _case("verify_bytes", "verify", 4, 4, 256, 0, "float32", rest=True),
        # one user, a large vocabulary: latency
        _case("verify_one", "verify", 1, 5, 131072, 0, "bfloat16"),
        # a serving batch, drafts of unequal lengths
        _case("verify_batch", "verify", 128, 8, 100003, 0, "bfloat16", "any", T=0.8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["top", "distill", "grad", "grad", "verify", "verify"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    while True:
        V = _log_int(rng, 16, 262144)
        if op == "verify":
            B, N, K = _log_int(rng, 1, 256), rng.randint(1, 8), 0
            rows = B * (2 * N + 1)
        else:
            B, N, K = _log_int(rng, 1, 32), _log_int(rng, 1, 4096), _log_int(rng, 1, min(V, 256))
            rows = B * N
        if rows * V <= (MAX_SORTED if op == "top" else MAX_ELEMENTS // 2):
            break
    rest = op != "top" and rng.random() < 0.5
    if rest and op != "verify":
        K = min(K, V // 2)                    # what is left has to be something
    c = _case("", op, B, N, V, K, dtype,
              lengths=rng.choice(["full", "any"] if op == "verify" else ["full", "half"]),
              pitch=V if rng.random() < 0.5 else (V + 63) // 64 * 64,
              rest=rest,
              ragged=op in ("distill", "grad") and rng.random() < 0.5,
              T=rng.choice([1.0, 1.0, 0.7, 2.0]))
    del c["name"]
    return c


# ---- inputs ----

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _lengths(case, seed):
    B, N = case["B"], case["N"]
    lo = {"full": N, "half": max(1, N // 2), "any": 0}[case["lengths"]]
    host = np.random.default_rng(seed).integers(lo, N, endpoint=True, size=B)
    return torch.from_numpy(host.astype(np.int32)).to(DEV)


def _places(g, shape, V, k):
    """k places of a row, no two of them alike."""
    step = V // k
    at = torch.randint(0, step, (*shape, k), generator=g, device=DEV)
    return at + torch.arange(k, device=DEV) * step


def _logits(g, B, N, case, places, values):
    """A language model's rows: most of the vocabulary in a broad bulk, a few tokens far above."""
    x = torch.randn((B, N, case["pitch"]), generator=g, device=DEV,
                    dtype=getattr(torch, case["dtype"]))
    x.mul_(2.0)
    x.scatter_(2, places, values.to(x.dtype))
    return x[..., :case["V"]]


def _peaks(g, shape, k):
    return 13.0 - 2.0 * torch.log1p(torch.arange(k, device=DEV)) + torch.randn(
        (*shape, k), generator=g, device=DEV)


def prepare(case, seed):
    op, B, N, V, K = case["op"], case["B"], case["N"], case["V"], case["K"]
    g = _generator(seed)
    st = {"case": case, "lengths": _lengths(case, seed)}
    if op == "verify":
        k = min(V, 16)
        x = _logits(g, B, N + 1, case, _places(g, (B, N + 1), V, k), _peaks(g, (B, N + 1), k))
        d = x[:, :N].float() + 0.7 * torch.randn((B, N, V), generator=g, device=DEV)
        if case["rest"]:
            d = d / case["T"]
            d = d - torch.logsumexp(d, 2, keepdim=True)
            st["draft_T"] = 1.0
        else:
            st["draft_T"] = case["T"]
        d = d.to(x.dtype)
        st["draft_lse"] = torch.logsumexp(d.float(), 2) if case["rest"] else None
        e = torch.empty((B, N, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
        st["tokens"] = (d.float() / st["draft_T"] - e.log_()).argmax(2).to(torch.int32)
        st["uniforms"] = torch.rand((B, N), generator=g, device=DEV)
        st["noise"] = torch.empty((B, V), device=DEV).exponential_(generator=g).clamp_(min=1e-30)
        st["target"], st["draft"] = x, d
        return st
    # a teacher's K largest logits, largest first, and the student's of the same tokens near them
    at = _places(g, (B, N), V, K)
    if op == "top":
        st["logits"] = _logits(g, B, N, case, at, _peaks(g, (B, N), K))
        return st
    t, order = _peaks(g, (B, N), K).sort(2, descending=True)
    at = at.gather(2, order)
    st["logits"] = _logits(g, B, N, case, at,
                           0.9 * t + 0.5 * torch.randn(t.shape, generator=g, device=DEV))
    t = t.to(st["logits"].dtype)
    if case["ragged"]:
        n = torch.randint(1, K + 1, (B, N, 1), generator=g, device=DEV)
        at = at.masked_fill(torch.arange(K, device=DEV) >= n, -1)
    st["values"], st["indices"] = t, at.to(torch.int32)
    st["weights"] = 0.5 + torch.rand((B, N), generator=g, device=DEV)
    st["lse"] = None
    if case["rest"]:
        left = 0.01 + 0.3 * torch.rand((B, N), generator=g, device=DEV)
        kept = (t.float() / case["T"]).masked_fill(at < 0, -math.inf)
        st["lse"] = torch.logsumexp(kept, 2) - torch.log1p(-left)
    return st


# ---- one pass ----

def run(state):
    return (_calls if own else _plain)(state)


def _calls(st):
    from paper_2002_00876_amd import binding

    case, n = st["case"], st["lengths"]
    op, T = case["op"], case["T"]
    if op == "top":
        return binding.top_logits(st["logits"], case["K"], n, temperature=T)
    if op == "distill":
        return binding.distill(st["logits"], st["values"], st["indices"], st["lse"], n,
                               temperature=T)
    if op == "grad":
        return binding.distill_grad(st["logits"], st["values"], st["indices"], st["lse"], n,
                                    weights=st["weights"], temperature=T)
    return binding.verify(st["target"], st["draft"], st["tokens"], st["uniforms"], st["noise"], n,
                          draft_lse=st["draft_lse"], temperature=T, draft_temperature=st["draft_T"])


def _lse(x):
    m = x.amax(-1, keepdim=True)
    return (m + (x - m).exp().sum(-1, keepdim=True).log()).squeeze(-1)


def _on(lengths, N):
    return torch.arange(N, device=DEV)[None] < lengths[:, None]


def _plain(st):
    op = st["case"]["op"]
    if op == "top":
        return _plain_top(st)
    return _plain_verify(st) if op == "verify" else _plain_distill(st)


def _plain_top(st):
    case, x = st["case"], st["logits"]
    on = _on(st["lengths"], case["N"])
    # equal logits: the lowest index first
    v, i = x.float().sort(dim=2, descending=True, stable=True)
    v, i = v[..., :case["K"]], i[..., :case["K"]].to(torch.int32)
    lse = _lse(x.float() / case["T"])
    return (v.masked_fill(~on[..., None], -math.inf).to(x.dtype), i.masked_fill(~on[..., None], -1),
            lse.masked_fill(~on, -math.inf))


def _plain_distill(st):
    case, at = st["case"], st["indices"].long()
    V, T = case["V"], case["T"]
    x = st["logits"].float() / T
    on, there = _on(st["lengths"], case["N"]), at >= 0
    t = (st["values"].float() / T).masked_fill(~there, -math.inf)
    logp = t - (_lse(t) if st["lse"] is None else st["lse"])[..., None]
    p = logp.exp()
    lse = _lse(x)
    logq = x.gather(2, at.clamp(min=0)) - lse[..., None]
    loss = torch.where(there, p * (logp - logq), 0.0).sum(2)
    low, keep = lse, torch.ones_like(lse)
    if st["lse"] is not None:
        top = torch.zeros((*x.shape[:2], V + 1), dtype=torch.bool, device=DEV)
        top.scatter_(2, torch.where(there, at, V), True)
        low = _lse(x.masked_fill(top[..., :V], -math.inf))
        left = 1.0 - p.sum(2)
        left = torch.where(left > MIN_REST, left, 0.0)
        more = left * (left.clamp(min=MIN_REST).log() - (low - lse))
        loss = loss + torch.where(left > 0, more, 0.0)
        keep = (low - lse).exp() - left
    loss = torch.where(on, loss, 0.0)
    if case["op"] == "distill":
        return loss
    scale = torch.where(on, st["weights"], 0.0) / T
    grad = torch.empty((*x.shape[:2], V + 1), device=DEV)
    torch.mul((x - low[..., None]).exp(), (scale * keep)[..., None], out=grad[..., :V])
    grad.scatter_(2, torch.where(there, at, V), scale[..., None] * (logq.exp() - p))
    return loss, grad[..., :V].to(st["logits"].dtype)


def _plain_verify(st):
    case = st["case"]
    B, G, V = case["B"], case["N"], case["V"]
    rows, n = torch.arange(B, device=DEV), st["lengths"].long()
    x = st["target"].float() / case["T"]
    y = st["draft"].float() / st["draft_T"]
    lx = _lse(x)
    ly = _lse(y) if st["draft_lse"] is None else st["draft_lse"]
    z = st["tokens"].long()
    p = (x[:, :G].gather(2, z[..., None])[..., 0] - lx[:, :G]).exp()
    q = (y.gather(2, z[..., None])[..., 0] - ly).exp()
    fails = ~(st["uniforms"] * q < p) | (torch.arange(G, device=DEV)[None] >= n[:, None])
    # the first position that fails, or the one after the last draft
    at = torch.arange(G + 1, device=DEV)
    stop = torch.cat([fails, torch.ones((B, 1), dtype=torch.bool, device=DEV)], 1)
    accepted = torch.where(stop, at[None], G).amin(1)
    pn = (x[rows, accepted] - lx[rows, accepted][:, None]).exp()
    at_q = accepted.clamp(max=max(G - 1, 0))
    qn = (y[rows, at_q] - ly[rows, at_q][:, None]).exp()
    left = torch.where((accepted < n)[:, None], (pn - qn).clamp(min=0), pn)
    left = torch.where((left > 0).any(1, keepdim=True), left, pn)
    score = left / st["noise"]
    best = score == score.amax(1, keepdim=True)                # equal scores: the lowest index
    new = torch.where(best, torch.arange(V, device=DEV)[None], V).amin(1)
    out = torch.cat([z, torch.zeros((B, 1), dtype=torch.int64, device=DEV)], 1)
    out = torch.where(at[None] < accepted[:, None], out, -1)
    out[rows, accepted] = new
    logp = x.gather(2, out.clamp(min=0)[..., None])[..., 0] - lx
    logp = torch.where(out >= 0, logp, 0.0)
    return out.to(torch.int32), accepted.to(torch.int32), logp


# ---- what a pass cannot do without ----

def work(case):
    B, N, V, K = case["B"], case["N"], case["V"], case["K"]
    size = 4 if case["dtype"] == "float32" else 2
    share = {"full": 1.0, "half": 0.75, "any": 0.5}[case["lengths"]]
    rows = B * N * share
    if case["op"] == "verify":
        # every draft accepted: all of the target's rows, the drafts' where they have to be
        # summed, and the last draw's noise; a maximum, an exponential and a sum a logit
        drafts = 1 if case["rest"] else V
        logits = B * (N * share + 1) * V + rows * drafts
        return {"bytes": int(logits * size + 4 * B * V + 8 * rows + 8 * B * (N + 1) + 4 * B),
                "flops": int(3 * logits + 4 * B * V)}
    logits = rows * V
    if case["op"] == "top":
        out = B * N * (K * (size + 4) + 4)
        return {"bytes": int(logits * size + out), "flops": int(4 * logits)}
    read = logits * size + rows * (K * (size + 4) + (4 if case["rest"] else 0))
    write, flops = 4 * B * N, 3 * logits + 8 * rows * K
    if case["op"] == "grad":                  # the gradient is written for padding too
        read, write, flops = read + 4 * rows, write + B * N * V * size, flops + 2 * logits
    return {"bytes": int(read + write), "flops": int(flops)}


# ---- the same results in float64 ----

def exact(case, seed):
    st = prepare(case, seed)
    B, N, V, n = case["B"], case["N"], case["V"], st["lengths"].tolist()
    if case["op"] == "verify":
        return _exact_verify(st, n)
    step = max(1, CHUNK // V)
    loss = torch.zeros((B, N), dtype=torch.float64, device=DEV)
    if case["op"] == "top":
        values = torch.full((B, N, case["K"]), -math.inf, dtype=torch.float64, device=DEV)
        lse = torch.full((B, N), -math.inf, dtype=torch.float64, device=DEV)
        for b in range(B):
            for s in range(0, n[b], step):
                e = min(n[b], s + step)
                x = st["logits"][b, s:e].double()
                values[b, s:e] = x.topk(case["K"], 1).values
                lse[b, s:e] = torch.logsumexp(x / case["T"], 1)
        return values, None, lse
    want = case["op"] == "grad"
    grad = torch.zeros((B, N, V), dtype=torch.float64, device=DEV) if want else None
    for b in range(B):
        for s in range(0, n[b], step):
            e = min(n[b], s + step)
            l, d = _exact_rows(st, b, s, e)
            loss[b, s:e] = l
            if want:
                grad[b, s:e] = d.mul_(st["weights"][b, s:e, None].double() / case["T"])
    return (loss, grad) if want else loss


def _exact_rows(st, b, s, e):
    """Loss and its derivative by the tempered logits, from dense distributions of both sides."""
    T = st["case"]["T"]
    logq = torch.log_softmax(st["logits"][b, s:e].double() / T, 1)
    at = st["indices"][b, s:e].long()
    t = torch.where(at >= 0, st["values"][b, s:e].double() / T, -math.inf)
    if st["lse"] is None:
        pk = torch.softmax(t, 1)
    else:
        pk = torch.exp(t - st["lse"][b, s:e, None].double())
    p = torch.zeros_like(logq)
    p.scatter_add_(1, at.clamp(min=0), pk)            # empty slots add nothing
    loss = (torch.special.xlogy(p, p) - p * logq).sum(1)
    q = logq.exp()
    d = q - p
    if st["lse"] is not None:
        slots = torch.zeros_like(q).scatter_add_(1, at.clamp(min=0), (at >= 0).double())
        rest = slots == 0
        q_rest, p_rest = torch.where(rest, q, 0.0).sum(1), 1.0 - pk.sum(1)
        loss = loss + torch.special.xlogy(p_rest, p_rest) - p_rest * q_rest.log()
        d = torch.where(rest, q * (1.0 - p_rest / q_rest)[:, None], d)
    return loss, d


def _exact_verify(st, n):
    case = st["case"]
    B, G = case["B"], case["N"]
    logps = torch.zeros((B, G + 1), dtype=torch.float64, device=DEV)
    for b in range(B):
        lp = torch.log_softmax(st["target"][b].double() / case["T"], 1)
        d = st["draft"][b].double() / st["draft_T"]
        lq = d - (torch.logsumexp(d, 1) if st["draft_lse"] is None
                  else st["draft_lse"][b].double())[:, None]
        z = st["tokens"][b].long()
        at = torch.arange(G, device=DEV)
        ok = (st["uniforms"][b].double().log() < lp[at, z] - lq[at, z]).tolist()
        a = 0
        while a < n[b] and ok[a]:
            a += 1
        left = lp[a].exp()
        if a < n[b]:
            left = (left - lq[a].exp()).clamp(min=0)
        new = (left / st["noise"][b].double()).argmax()
        logps[b, :a] = lp[at[:a], z[:a]]
        logps[b, a] = lp[a, new]
    return None, None, logps
