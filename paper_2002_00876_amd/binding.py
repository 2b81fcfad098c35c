"""Python binding of libtschain.so: marshals torch tensors (device memory and the
current HIP stream) into the C ABI of include/ts_chain.h and include/ts_token.h.  No arithmetic happens here;
every step runs in the library's HIP kernels.  If the library is missing, every call
raises: there is no fallback."""
import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libtschain.so")

OP_LOGPARTITION, OP_MARGINALS, OP_VITERBI, OP_MARGINALS_VITERBI = 0, 1, 2, 3
OP_ENTROPY, OP_LOG_DENSITY, OP_SAMPLE = 4, 5, 6
TOKEN_TOP, TOKEN_DISTILL, TOKEN_DISTILL_GRAD, TOKEN_VERIFY = 0, 1, 2, 3
STATUS = {0: "TS_OK", -1: "TS_ERR_NULL_ARG", -2: "TS_ERR_BAD_DIM", -3: "TS_ERR_WORKSPACE",
          -4: "TS_ERR_LENGTHS", -5: "TS_ERR_HIP", -6: "TS_ERR_LABELS",
          -7: "TS_ERR_BAD_ARG"}
DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}

_lib = None


class TsError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


def lib():
    """The loaded C library with argument types declared (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run paper_2002_00876_amd.build.build()")
        L = ctypes.CDLL(LIB_PATH)
        i64, p, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
        L.ts_chain_max_labels.restype = ctypes.c_int
        L.ts_chain_workspace_bytes.argtypes = [ctypes.c_int, i64, i64, i64]
        L.ts_chain_workspace_bytes.restype = sz
        L.ts_chain_logpartition.argtypes = [p, p, i64, i64, i64, p, p, sz, p]
        L.ts_chain_marginals.argtypes = [p, p, i64, i64, i64, p, p, p, sz, p]
        L.ts_chain_viterbi.argtypes = [p, p, i64, i64, i64, p, p, p, sz, p]
        L.ts_chain_marginals_viterbi.argtypes = [p, p, i64, i64, i64, p, p, p, p, p, sz, p]
        L.ts_chain_marginals_noalloc.argtypes = [p, p, i64, i64, i64, p, p, p]
        L.ts_chain_noalloc_scratch_bytes.restype = sz
        L.ts_chain_entropy.argtypes = [p, p, i64, i64, i64, p, p, sz, p]
        L.ts_chain_log_density.argtypes = [p, p, p, i64, i64, i64, p, p, sz, p]
        L.ts_chain_logpartition_sequential.argtypes = [p, p, i64, i64, i64, p, p]
        L.ts_chain_sample.argtypes = [p, p, p, i64, i64, i64, i64, p, p, sz, p]
        L.ts_semimarkov_workspace_bytes.argtypes = [ctypes.c_int, i64, i64, i64, i64]
        L.ts_semimarkov_workspace_bytes.restype = sz
        L.ts_semimarkov_logpartition.argtypes = [p, p, i64, i64, i64, i64, p, p, sz, p]
        L.ts_semimarkov_marginals.argtypes = [p, p, i64, i64, i64, i64, p, p, p, sz, p]
        L.ts_semimarkov_viterbi.argtypes = [p, p, i64, i64, i64, i64, p, p, p, p, sz, p]
        f32, ci = ctypes.c_float, ctypes.c_int
        L.ts_token_max_vocab.restype = ci
        L.ts_token_max_top.restype = ci
        L.ts_token_workspace_bytes.argtypes = [ci, i64, i64, i64, i64]
        L.ts_token_workspace_bytes.restype = sz
        L.ts_token_top.argtypes = [p, ci, i64, i64, p, i64, i64, i64, i64, f32, p, p, p, p, sz, p]
        L.ts_token_distill.argtypes = [p, ci, i64, i64, p, ci, p, p, p, i64, i64, i64, i64, f32, p,
                                       p, sz, p]
        L.ts_token_distill_grad.argtypes = [p, ci, i64, i64, p, ci, p, p, p, p, i64, i64, i64, i64,
                                            f32, p, p, p, sz, p]
        L.ts_token_verify.argtypes = [p, ci, i64, i64, p, ci, i64, i64, p, p, p, p, p, i64, i64,
                                      i64, f32, f32, p, p, p, p, sz, p]
        for f in ("ts_token_top", "ts_token_distill", "ts_token_distill_grad", "ts_token_verify",
                  "ts_chain_logpartition", "ts_chain_marginals", "ts_chain_viterbi",
                  "ts_chain_marginals_noalloc",
                  "ts_chain_marginals_viterbi", "ts_chain_entropy", "ts_chain_log_density",
                  "ts_chain_logpartition_sequential", "ts_chain_sample",
                  "ts_semimarkov_logpartition", "ts_semimarkov_marginals",
                  "ts_semimarkov_viterbi"):
            getattr(L, f).restype = ctypes.c_int
        L.ts_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(code):
    if code != 0:
        raise TsError(code, lib().ts_last_error().decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(device):
    # the current stream's handle without a Stream object around it (0.2 instead of 2.0 us, of
    # the 9 us that a smallest call takes on the host)
    return torch._C._cuda_getCurrentRawStream(device.index)


def _prep(pot, lengths):
    if not pot.is_cuda:
        raise ValueError("pot must be a device tensor")
    if pot.dtype != torch.float32 or pot.dim() != 4 or pot.shape[2] != pot.shape[3]:
        raise ValueError("pot must be float32 [B, N-1, C, C]")
    pot = pot.contiguous()
    B, E, C, _ = pot.shape
    if lengths is not None:
        if lengths.device != pot.device or lengths.dtype != torch.int32 or lengths.shape != (B,):
            raise ValueError("lengths must be int32 [B] on the same device as pot")
        lengths = lengths.contiguous()
    return pot, lengths, B, E + 1, C


def workspace_bytes(op, B, N, C):
    return lib().ts_chain_workspace_bytes(op, B, N, C)


def _workspace(op, B, N, C, device, ws=None):
    need = workspace_bytes(op, B, N, C)
    if ws is not None:
        return ws, ws.numel() * ws.element_size()
    if need == 0:
        return None, 0
    return torch.empty(need, dtype=torch.uint8, device=device), need


def logpartition(pot, lengths=None, out=None, ws=None):
    """log Z [B] (float32) of potentials [B, N-1, C, C] with token lengths [B]."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    logz = out if out is not None else torch.empty(B, dtype=torch.float32, device=pot.device)
    w, nb = _workspace(OP_LOGPARTITION, B, N, C, pot.device, ws)
    _check(lib().ts_chain_logpartition(_ptr(pot), _ptr(lengths), B, N, C, _ptr(logz), _ptr(w),
                                       nb, _stream(pot.device)))
    return logz


def marginals(pot, lengths=None, out=None, ws=None, want_logz=True):
    """(log Z [B] or None, edge marginals [B, N-1, C, C]), float32."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    if out is not None:
        logz, marg = out
    else:
        logz = torch.empty(B, dtype=torch.float32, device=pot.device) if want_logz else None
        marg = torch.empty_like(pot)
    w, nb = _workspace(OP_MARGINALS, B, N, C, pot.device, ws)
    _check(lib().ts_chain_marginals(_ptr(pot), _ptr(lengths), B, N, C, _ptr(logz),
                                    _ptr(marg) if N > 1 else None, _ptr(w), nb,
                                    _stream(pot.device)))
    return logz, marg


def noalloc_scratch_bytes():
    """Bytes of the per-GPU scratch array of the allocation-free marginals call."""
    return lib().ts_chain_noalloc_scratch_bytes()


def marginals_noalloc(pot, lengths=None, out=None, want_logz=True):
    """marginals() through ts_chain_marginals_noalloc: no workspace; the library's per-GPU
    scratch array is used instead (calls on one GPU must not overlap)."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    if out is not None:
        logz, marg = out
    else:
        logz = torch.empty(B, dtype=torch.float32, device=pot.device) if want_logz else None
        marg = torch.empty_like(pot)
    _check(lib().ts_chain_marginals_noalloc(_ptr(pot), _ptr(lengths), B, N, C, _ptr(logz),
                                            _ptr(marg) if N > 1 else None,
                                            _stream(pot.device)))
    return logz, marg


def viterbi(pot, lengths=None, out=None, ws=None):
    """(path int32 [B, N] with -1 past each length, score float32 [B])."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    if out is not None:
        path, score = out
    else:
        path = torch.empty((B, N), dtype=torch.int32, device=pot.device)
        score = torch.empty(B, dtype=torch.float32, device=pot.device)
    w, nb = _workspace(OP_VITERBI, B, N, C, pot.device, ws)
    _check(lib().ts_chain_viterbi(_ptr(pot), _ptr(lengths), B, N, C, _ptr(path), _ptr(score),
                                  _ptr(w), nb, _stream(pot.device)))
    return path, score


def marginals_viterbi(pot, lengths=None, out=None, ws=None, want_logz=True):
    """(log Z [B] or None, marginals [B, N-1, C, C], path [B, N], score [B]) in one call."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    if out is not None:
        logz, marg, path, score = out
    else:
        dev = pot.device
        logz = torch.empty(B, dtype=torch.float32, device=dev) if want_logz else None
        marg = torch.empty_like(pot)
        path = torch.empty((B, N), dtype=torch.int32, device=dev)
        score = torch.empty(B, dtype=torch.float32, device=dev)
    w, nb = _workspace(OP_MARGINALS_VITERBI, B, N, C, pot.device, ws)
    _check(lib().ts_chain_marginals_viterbi(_ptr(pot), _ptr(lengths), B, N, C, _ptr(logz),
                                            _ptr(marg) if N > 1 else None, _ptr(path),
                                            _ptr(score), _ptr(w), nb, _stream(pot.device)))
    return logz, marg, path, score


def entropy(pot, lengths=None, out=None, ws=None):
    """Entropy [B] (float32) of each sequence's label distribution."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    h = out if out is not None else torch.empty(B, dtype=torch.float32, device=pot.device)
    w, nb = _workspace(OP_ENTROPY, B, N, C, pot.device, ws)
    _check(lib().ts_chain_entropy(_ptr(pot), _ptr(lengths), B, N, C, _ptr(h), _ptr(w), nb,
                                  _stream(pot.device)))
    return h


def log_density(pot, labels, lengths=None, out=None, ws=None):
    """log p(z) [B] (float32) of label sequences labels (int32 [B, N])."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    if labels.device != pot.device or labels.dtype != torch.int32 or labels.shape != (B, N):
        raise ValueError("labels must be int32 [B, N] on the same device as pot")
    labels = labels.contiguous()
    lp = out if out is not None else torch.empty(B, dtype=torch.float32, device=pot.device)
    w, nb = _workspace(OP_LOG_DENSITY, B, N, C, pot.device, ws)
    _check(lib().ts_chain_log_density(_ptr(pot), _ptr(lengths), _ptr(labels), B, N, C, _ptr(lp),
                                      _ptr(w), nb, _stream(pot.device)))
    return lp


def logpartition_sequential(pot, lengths=None, out=None):
    """log Z [B] by the left-to-right forward algorithm (the serial baseline of the scan)."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    logz = out if out is not None else torch.empty(B, dtype=torch.float32, device=pot.device)
    _check(lib().ts_chain_logpartition_sequential(_ptr(pot), _ptr(lengths), B, N, C, _ptr(logz),
                                                  _stream(pot.device)))
    return logz


def sample(pot, uniforms, lengths=None, out=None, ws=None):
    """Forward-filtering backward-sampling draws: paths int32 [S, B, N] (-1 past each
    length) from caller-supplied uniforms float32 [S, B, N] in [0, 1)."""
    pot, lengths, B, N, C = _prep(pot, lengths)
    if (uniforms.device != pot.device or uniforms.dtype != torch.float32 or uniforms.dim() != 3
            or tuple(uniforms.shape[1:]) != (B, N)):
        raise ValueError("uniforms must be float32 [S, B, N] on the same device as pot")
    uniforms = uniforms.contiguous()
    S = uniforms.shape[0]
    paths = out if out is not None else torch.empty((S, B, N), dtype=torch.int32,
                                                    device=pot.device)
    w, nb = _workspace(OP_SAMPLE, B, N, C, pot.device, ws)
    _check(lib().ts_chain_sample(_ptr(pot), _ptr(lengths), _ptr(uniforms), S, B, N, C,
                                 _ptr(paths), _ptr(w), nb, _stream(pot.device)))
    return paths


# ---- semi-Markov CRF: segment potentials sp [B, N-1, K, C, C] ----

def _prep_semi(sp, lengths):
    if not sp.is_cuda:
        raise ValueError("sp must be a device tensor")
    if sp.dtype != torch.float32 or sp.dim() != 5 or sp.shape[3] != sp.shape[4]:
        raise ValueError("sp must be float32 [B, N-1, K, C, C]")
    sp = sp.contiguous()
    B, E, K, C, _ = sp.shape
    if lengths is not None:
        if lengths.device != sp.device or lengths.dtype != torch.int32 or lengths.shape != (B,):
            raise ValueError("lengths must be int32 [B] on the same device as sp")
        lengths = lengths.contiguous()
    return sp, lengths, B, E + 1, K, C


def semi_workspace_bytes(op, B, N, K, C):
    return lib().ts_semimarkov_workspace_bytes(op, B, N, K, C)


def _semi_workspace(op, B, N, K, C, device, ws=None):
    if ws is not None:
        return ws, ws.numel() * ws.element_size()
    need = semi_workspace_bytes(op, B, N, K, C)
    if need == 0:
        return None, 0
    return torch.empty(need, dtype=torch.uint8, device=device), need


def semi_logpartition(sp, lengths=None, out=None, ws=None):
    """Semi-Markov log Z [B] (float32)."""
    sp, lengths, B, N, K, C = _prep_semi(sp, lengths)
    logz = out if out is not None else torch.empty(B, dtype=torch.float32, device=sp.device)
    w, nb = _semi_workspace(OP_LOGPARTITION, B, N, K, C, sp.device, ws)
    _check(lib().ts_semimarkov_logpartition(_ptr(sp), _ptr(lengths), B, N, K, C, _ptr(logz),
                                            _ptr(w), nb, _stream(sp.device)))
    return logz


def semi_marginals(sp, lengths=None, out=None, ws=None, want_logz=True):
    """Semi-Markov (log Z [B] or None, segment marginals [B, N-1, K, C, C]), float32."""
    sp, lengths, B, N, K, C = _prep_semi(sp, lengths)
    if out is not None:
        logz, marg = out
    else:
        logz = torch.empty(B, dtype=torch.float32, device=sp.device) if want_logz else None
        marg = torch.empty_like(sp)
    w, nb = _semi_workspace(OP_MARGINALS, B, N, K, C, sp.device, ws)
    _check(lib().ts_semimarkov_marginals(_ptr(sp), _ptr(lengths), B, N, K, C, _ptr(logz),
                                         _ptr(marg) if N > 1 else None, _ptr(w), nb,
                                         _stream(sp.device)))
    return logz, marg


def semi_viterbi(sp, lengths=None, out=None, ws=None):
    """Semi-Markov best segmentation: (path int32 [B, N], seglen int32 [B, N-1],
    score float32 [B])."""
    sp, lengths, B, N, K, C = _prep_semi(sp, lengths)
    if out is not None:
        path, seglen, score = out
    else:
        dev = sp.device
        path = torch.empty((B, N), dtype=torch.int32, device=dev)
        seglen = torch.empty((B, N - 1), dtype=torch.int32, device=dev)
        score = torch.empty(B, dtype=torch.float32, device=dev)
    w, nb = _semi_workspace(OP_VITERBI, B, N, K, C, sp.device, ws)
    _check(lib().ts_semimarkov_viterbi(_ptr(sp), _ptr(lengths), B, N, K, C, _ptr(path),
                                       _ptr(seglen) if N > 1 else None, _ptr(score), _ptr(w),
                                       nb, _stream(sp.device)))
    return path, seglen, score


# ---- rows of token logits [B, N, V] (include/ts_token.h) ----

def _prep_rows(x, name):
    """x with its rows contiguous (copied only where they are not), its type's code and the
    elements from a sequence, a row to the next."""
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if x.dtype not in DTYPES or x.dim() != 3:
        raise ValueError(f"{name} must be float32, bfloat16 or float16 [B, N, V]")
    if x.shape[2] > 1 and x.stride(2) != 1:
        x = x.contiguous()
    return x, DTYPES[x.dtype], x.stride(0), x.stride(1)


def _prep_small(x, name, dtype, shape, device):
    if x is None:
        return None
    if x.dtype != dtype or x.shape != shape or x.device != device:
        raise ValueError(f"{name} must be {dtype} {list(shape)} on the same device as the logits")
    return x if x.is_contiguous() else x.contiguous()


def _check_outs(out, names, dtypes, shapes, device):
    if len(out) != len(names):
        raise ValueError(f"out must be ({', '.join(names)})")
    for x, name, dtype, shape in zip(out, names, dtypes, shapes):
        if x.dtype != dtype or x.shape != shape or x.device != device or not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dtype} {list(shape)} on the same device "
                             "as the logits")
    return out


def token_workspace_bytes(op, B, N, V, K=1):
    return lib().ts_token_workspace_bytes(op, B, N, V, K)


def _token_workspace(op, B, N, V, K, device, ws):
    if ws is not None:
        if ws.device != device or not ws.is_contiguous():
            raise ValueError("ws must be a contiguous tensor on the same device as the logits")
        return ws, ws.numel() * ws.element_size()
    need = token_workspace_bytes(op, B, N, V, K)
    if need == 0:
        return None, 0
    return torch.empty(need, dtype=torch.uint8, device=device), need


def top_logits(logits, K, lengths=None, temperature=1.0, out=None, ws=None):
    """(values [B, N, K] of the logits' type, indices int32 [B, N, K], lse float32 [B, N]): the K
    largest logits of every row of logits [B, N, V], largest first and equal ones by the lowest
    index, and log sum exp(logits / temperature).  Rows from lengths (int32 [B]) on are padding:
    values and lse -inf, indices -1."""
    logits, dtype, sb, sn = _prep_rows(logits, "logits")
    B, N, V = logits.shape
    dev = logits.device
    lengths = _prep_small(lengths, "lengths", torch.int32, (B,), dev)
    if out is None:
        values = torch.empty((B, N, K), dtype=logits.dtype, device=dev)
        indices = torch.empty((B, N, K), dtype=torch.int32, device=dev)
        lse = torch.empty((B, N), dtype=torch.float32, device=dev)
    else:
        values, indices, lse = _check_outs(
            out, ("values", "indices", "lse"), (logits.dtype, torch.int32, torch.float32),
            ((B, N, K), (B, N, K), (B, N)), dev)
    w, nb = _token_workspace(TOKEN_TOP, B, N, V, K, dev, ws)
    _check(lib().ts_token_top(_ptr(logits), dtype, sb, sn, _ptr(lengths), B, N, V, K, temperature,
                              _ptr(values), _ptr(indices), _ptr(lse), _ptr(w), nb, _stream(dev)))
    return values, indices, lse


def _prep_teacher(logits, top_values, top_indices, top_lse, lengths):
    logits, dtype, sb, sn = _prep_rows(logits, "logits")
    B, N, V = logits.shape
    dev = logits.device
    if top_values.dtype not in DTYPES or top_values.dim() != 3:
        raise ValueError("top_values must be float32, bfloat16 or float16 [B, N, K]")
    K = top_values.shape[2]
    top_values = _prep_small(top_values, "top_values", top_values.dtype, (B, N, K), dev)
    top_indices = _prep_small(top_indices, "top_indices", torch.int32, (B, N, K), dev)
    top_lse = _prep_small(top_lse, "top_lse", torch.float32, (B, N), dev)
    lengths = _prep_small(lengths, "lengths", torch.int32, (B,), dev)
    head = (_ptr(logits), dtype, sb, sn, _ptr(top_values), DTYPES[top_values.dtype],
            _ptr(top_indices), _ptr(top_lse))
    # the tensors themselves are returned too: copies made here have to outlive the launch
    return head, (logits, top_values, top_indices, top_lse, lengths), (B, N, V, K), dev


def distill(logits, top_values, top_indices, top_lse=None, lengths=None, temperature=1.0, out=None,
            ws=None):
    """Kullback-Leibler divergence [B, N] (float32) of softmax(logits / temperature), logits
    [B, N, V], from a teacher's top logits: values [B, N, K] at indices int32 [B, N, K] (an index
    outside the vocabulary is an empty slot).  Without top_lse the teacher is normalised over
    its slots; with it (its log-sum-exp [B, N] at this temperature) what they leave is one class.
    0 for padding.  The loss has no graph: distill_grad() is its backward pass."""
    head, kept, (B, N, V, K), dev = _prep_teacher(logits, top_values, top_indices, top_lse, lengths)
    if out is None:
        loss = torch.empty((B, N), dtype=torch.float32, device=dev)
    else:
        loss, = _check_outs((out,), ("loss",), (torch.float32,), ((B, N),), dev)
    w, nb = _token_workspace(TOKEN_DISTILL, B, N, V, K, dev, ws)
    _check(lib().ts_token_distill(*head, _ptr(kept[-1]), B, N, V, K, temperature, _ptr(loss),
                                  _ptr(w), nb, _stream(dev)))
    return loss


def distill_grad(logits, top_values, top_indices, top_lse=None, lengths=None, weights=None,
                 temperature=1.0, out=None, ws=None, want_loss=True):
    """(loss [B, N] or None as distill()'s, grad [B, N, V] of the logits' type): the gradient of
    sum(weights * loss) by the logits, weights float32 [B, N] (None: all 1)."""
    head, kept, (B, N, V, K), dev = _prep_teacher(logits, top_values, top_indices, top_lse, lengths)
    weights = _prep_small(weights, "weights", torch.float32, (B, N), dev)
    if out is None:
        loss = torch.empty((B, N), dtype=torch.float32, device=dev) if want_loss else None
        grad = torch.empty((B, N, V), dtype=logits.dtype, device=dev)
    else:
        loss, grad = _check_outs(out, ("loss", "grad"), (torch.float32, logits.dtype),
                                 ((B, N), (B, N, V)), dev)
    w, nb = _token_workspace(TOKEN_DISTILL_GRAD, B, N, V, K, dev, ws)
    _check(lib().ts_token_distill_grad(*head, _ptr(weights), _ptr(kept[-1]), B, N, V, K,
                                       temperature, _ptr(loss) if want_loss else None, _ptr(grad),
                                       _ptr(w), nb, _stream(dev)))
    return (loss if want_loss else None), grad


def verify(target, draft, tokens, uniforms, noise, lengths=None, draft_lse=None, temperature=1.0,
           draft_temperature=1.0, out=None, ws=None):
    """(out int32 [B, G+1], accepted int32 [B], logp float32 [B, G+1]): the drafts tokens (int32
    [B, G]) that the target's probabilities accept, then one more token, then -1; the number of
    accepted ones; the target's log-probabilities of what is emitted.  target [B, G+1, V] and
    draft [B, G, V] are logits, draft_lse [B, G] the drafts' log-sum-exps where they are known
    (0 for log-probabilities), uniforms float32 [B, G] in [0, 1) and noise float32 [B, V]
    (standard exponentials) the caller's random numbers, lengths (int32 [B]) the drafts of each
    sequence."""
    target, dtype, sb, sn = _prep_rows(target, "target")
    B, G, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    dev = target.device
    draft, ddtype, db, dn = _prep_rows(draft, "draft")
    if draft.shape != (B, G, V) or draft.device != dev:
        raise ValueError(f"draft must be {[B, G, V]} on the same device as the target")
    tokens = _prep_small(tokens, "tokens", torch.int32, (B, G), dev)
    uniforms = _prep_small(uniforms, "uniforms", torch.float32, (B, G), dev)
    noise = _prep_small(noise, "noise", torch.float32, (B, V), dev)
    draft_lse = _prep_small(draft_lse, "draft_lse", torch.float32, (B, G), dev)
    lengths = _prep_small(lengths, "lengths", torch.int32, (B,), dev)
    if out is None:
        emitted = torch.empty((B, G + 1), dtype=torch.int32, device=dev)
        accepted = torch.empty(B, dtype=torch.int32, device=dev)
        logp = torch.empty((B, G + 1), dtype=torch.float32, device=dev)
    else:
        emitted, accepted, logp = _check_outs(
            out, ("out", "accepted", "logp"), (torch.int32, torch.int32, torch.float32),
            ((B, G + 1), (B,), (B, G + 1)), dev)
    w, nb = _token_workspace(TOKEN_VERIFY, B, G, V, 1, dev, ws)
    _check(lib().ts_token_verify(_ptr(target), dtype, sb, sn, _ptr(draft), ddtype, db, dn,
                                 _ptr(draft_lse), _ptr(tokens), _ptr(uniforms), _ptr(noise),
                                 _ptr(lengths), B, G, V, temperature, draft_temperature,
                                 _ptr(emitted), _ptr(accepted), _ptr(logp), _ptr(w), nb,
                                 _stream(dev)))
    return emitted, accepted, logp
