"""A larger model's pass over a chain's drafts, call after call as a program makes them: the text into
the cache, drafts sampled from the chain, their keys and values behind it, attention over all, the
verification of the drafts and the scores of what is emitted, and a step of the model's head on that.
The model (one layer of attention) is computed in float64 from whole sequences beside it."""
import numpy as np
import pytest

import cache_ref
import token_ref
from gpu_util import say

pytestmark = pytest.mark.gpu

V, Hq, Hk, D, S, G = 24, 4, 2, 64, 16, 4
FREQS = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)


class Model:
    """Tokens' queries, keys and values by three tables, logits by a matrix; all of them bfloat16."""

    def __init__(self, seed):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        table = lambda h: torch.randn((V, h, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        self.q, self.k, self.v = table(Hq), table(Hk), table(Hk)
        self.head = torch.randn((Hq * D, V), generator=g, device="cuda")

    def check(self, b, tokens, positions, i, n, q, out, kc, vc, pages, starts, parents):
        """A sequence's cache holds its tokens' keys and values at their positions, the last n of them the
        pass's; its queries (rows i of the call) and the attention's rows are theirs: each of the calls
        within its own bounds, given what the one before left."""
        rows = lambda t: t.double().cpu().numpy()[tokens]  # noqa: E731
        host = lambda t: t.double().nan_to_num().cpu().numpy()  # noqa: E731
        kc, vc, q, out = host(kc), host(vc), host(q), host(out)
        pages, total = pages.cpu().numpy(), len(tokens)
        k, off = cache_ref.rotate(rows(self.k), np.asarray(positions), FREQS, False, "bfloat16")
        assert (np.abs(cache_ref.slots(kc, pages, S, b, total) - k) <= off).all()
        assert np.array_equal(cache_ref.slots(vc, pages, S, b, total), rows(self.v))
        want, off = cache_ref.rotate(rows(self.q), np.asarray(positions), FREQS, False, "bfloat16")
        assert (np.abs(q[b, i] - want[total - n:]) <= off[total - n:]).all()
        one = slice(b, b + 1)
        want, _, off, _ = cache_ref.attend(q[one], kc, vc, pages[one], [total - n], [n],
                                           None if parents is None else parents[one], D ** -0.5, "bfloat16")
        assert (np.abs(out[b, i] - want[0, i]) <= off[0, i]).all()


def _ints(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _setup(seed, B, room):
    """A model, a chain over its tokens, texts in the cache, and the last token of each not yet."""
    import torch
    from paper_2002_00876_amd import binding
    rng = np.random.default_rng(seed)
    model = Model(seed)
    lens = rng.integers(1, 60, size=B)
    texts = [rng.integers(0, V, size=n) for n in lens]
    N = int(lens.max())
    padded = np.zeros((B, N), dtype=np.int64)
    for b, t in enumerate(texts):
        padded[b, :len(t)] = t
    M = -(-(N + room) // S)
    P = B * M + 1
    pages = _ints(rng.permutation(P)[:B * M].reshape(B, M))
    kc, vc = (torch.full((P, S, Hk, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    at = torch.from_numpy(padded).cuda()
    binding.cache_append(model.k[at], model.v[at], kc, vc, pages, _ints(np.zeros(B)), _ints(lens - 1),
                         freqs=torch.from_numpy(FREQS).cuda())
    return rng, model, texts, lens, pages, kc, vc


def _pass(model, tokens, kc, vc, pages, starts, parents=None, positions=None, lengths=None):
    """The model's logits of tokens [B, N] behind what the cache holds."""
    import torch
    from paper_2002_00876_amd import binding
    at = tokens.long()
    q = binding.cache_append(model.k[at], model.v[at], kc, vc, pages, starts, lengths, q=model.q[at],
                             freqs=torch.from_numpy(FREQS).cuda(), positions=positions)
    out, _ = binding.tree_attention(q, kc, vc, pages, starts, parents, lengths)
    return (out.reshape(*at.shape, Hq * D).float() @ model.head), q, out


@pytest.mark.parametrize("seed", [0, 1, 2])
def test_drafts_of_a_chain(seed):
    import torch
    from paper_2002_00876_amd import binding
    B = 5
    rng, model, texts, lens, pages, kc, vc = _setup(seed, B, G + 1)
    # the chain: its first label is the text's last token, what follows is drafted
    pot = torch.from_numpy(rng.normal(0, 1, size=(B, G, V, V)).astype(np.float32)).cuda()
    first = torch.full((B, V), -float("inf"), device="cuda")
    first[torch.arange(B), torch.tensor([t[-1] for t in texts], device="cuda")] = 0.0
    pot[:, 0] += first[:, :, None]
    path = binding.sample(pot, torch.from_numpy(rng.random((1, B, G + 1), dtype=np.float32)).cuda())[0]
    assert path[:, 0].tolist() == [t[-1] for t in texts]
    logits, turned, rows_out = _pass(model, path, kc, vc, pages, _ints(lens - 1))
    # q_t: the chain's next-label probabilities, from its own backward messages
    back, rows = torch.zeros((B, V), device="cuda", dtype=torch.float64), []
    for t in range(G - 1, -1, -1):
        rows.append(pot[:, t].double() + back[:, None])
        back = torch.logsumexp(rows[-1], 2)
    z = path.long()
    draft = torch.stack([torch.log_softmax(rows[G - 1 - t][torch.arange(B), z[:, t]], 1)
                         for t in range(G)], 1).float()
    u = torch.from_numpy(rng.random((B, G), dtype=np.float32)).cuda()
    e = torch.from_numpy(rng.exponential(size=(B, V)).astype(np.float32)).cuda()
    out, accepted, logp = binding.verify(logits, draft, path[:, 1:].contiguous(), u, e,
                                         draft_lse=torch.zeros((B, G), device="cuda"))
    scored, entropy, best, best_lp = binding.score(logits, out, 3)
    torch.cuda.synchronize()
    x, d = logits.double().cpu().numpy(), draft.double().cpu().numpy()
    for b in range(B):
        whole = np.concatenate([texts[b], path[b, 1:].cpu().numpy()])
        model.check(b, whole, np.arange(len(whole)), slice(None), G + 1, turned, rows_out, kc, vc, pages,
                    lens - 1, None)
        emitted, a, lp, margin = token_ref.verify(x[b], d[b], path[b, 1:].cpu().numpy(),
                                                  u[b].cpu().numpy(), e[b].double().cpu().numpy(), G, 1.0,
                                                  1.0, np.zeros(G))
        if margin > 1e-4:
            assert out[b, :a + 1].tolist() == emitted and int(accepted[b]) == a
        n = int(accepted[b]) + 1
        assert torch.allclose(scored[b, :n], logp[b, :n], atol=1e-5) and (scored[b, n:] == 0).all()
        p = torch.softmax(logits[b].double(), 1)
        assert torch.allclose(entropy[b].double(), -(p * p.log()).sum(1), atol=1e-4)
        assert best[b, :, 0].tolist() == logits[b].argmax(1).tolist()
        assert (best_lp[b, :, 0] >= best_lp[b, :, 1]).all()
    # the head's step on what was emitted, against the same by the graph of plain operations
    n = accepted + 1
    w = torch.where(torch.arange(G + 1, device="cuda")[None] < n[:, None], -1.0 / float(n.sum()), 0.0)
    _, _, g = binding.score_grad(logits, out, n, weights=w, entropy_weights=w * 0.1)
    y = logits.double().requires_grad_()
    lp = torch.log_softmax(y, 2)
    h = -(lp.exp() * lp).sum(2)
    chosen = lp.gather(2, out.clamp(min=0).long()[..., None])[..., 0]
    (w * chosen + 0.1 * w * h).sum().backward()
    assert torch.allclose(g.double(), y.grad, atol=1e-6)


@pytest.mark.parametrize("seed", [3, 4])
def test_a_tree_of_samples_is_its_paths(seed):
    """Samples of a chain merged where they begin alike: each node's row is that of its own path."""
    import torch
    B, samples = 3, 6
    rng, model, texts, lens, pages, kc, vc = _setup(seed, B, 1 + samples * G)
    nodes, paths = [], []
    for b in range(B):
        at = {(): 0}
        own, mine = [(int(texts[b][-1]), -1, 0)], []
        for _ in range(samples):
            key, where = (), []
            for t in rng.integers(0, 3, size=G):        # few labels: shared beginnings
                up, key = at[key], key + (int(t),)
                if key not in at:
                    at[key] = len(own)
                    own.append((int(t), up, len(key)))
                where.append(at[key])
            mine.append(where)
        nodes.append(own)
        paths.append(mine)
    n = [len(x) for x in nodes]
    N = max(n)
    tok, par, dep = (np.array([[x[i][f] if i < len(x) else 0 for i in range(N)] for x in nodes])
                     for f in range(3))
    say(f"tree of {n} nodes")
    starts = _ints(lens - 1)
    _, turned, tree = _pass(model, _ints(tok), kc, vc, pages, starts, _ints(par),
                            _ints(dep + (lens - 1)[:, None]), _ints(n))
    for b in range(B):
        whole = np.concatenate([texts[b][:-1], tok[b, :n[b]]])
        at = np.concatenate([np.arange(lens[b] - 1), lens[b] - 1 + dep[b, :n[b]]])
        model.check(b, whole, at, slice(0, n[b]), n[b], turned, tree, kc, vc, pages, lens - 1, par)
        assert (tree[b, n[b]:] == 0).all()
    # a path's own pass sees the same keys and values in another order: each side within its own bounds of
    # the same sums, which the first of them says
    for s in range(samples):
        one = _ints([[x[0][0]] + [x[i][0] for i in p[s]] for x, p in zip(nodes, paths)])
        _, q, out = _pass(model, one, kc, vc, pages, starts)
        path = np.arange(-1, G)[None].repeat(B, 0)
        for b in range(B):
            whole = np.concatenate([texts[b], one[b, 1:].cpu().numpy()])
            model.check(b, whole, np.arange(len(whole)), slice(None), G + 1, q, out, kc, vc, pages, lens - 1,
                        path)
            rows = [0] + paths[b][s]
            assert torch.equal(q[b], turned[b, rows])
            size = float(model.v.abs().max())       # of a mean of values: half a step of each of both
            assert (out[b].float() - tree[b, rows].float()).abs().max() <= 4 * 2.0 ** -8 * size + 1e-4
