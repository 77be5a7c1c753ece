"""Plain 64-bit references of the decoding calls (qnn_linear_attention, qnn_beam_select, qnn_beam_reorder, qnn_embedding,
qnn_embedding_grad), with the error bounds their fp32 forms are held to. numpy only.

u = 2^-24 is the largest relative error of one fp32 rounding. A matrix instruction adds its products to its sum cut off, by 2 u of the
largest term at most.
"""
from __future__ import annotations

import numpy as np

from layer_ref import HALF, TINY, U


def heads(x, H):
    return np.repeat(x, H // x.shape[2], 2).astype(np.float64)


def linear(q, k, v, log_decay, scale, kind, state=None, lengths=None):
    """(y, bound, state, bound): q, k [B, T, heads, dk], v [B, T, heads, dv]; frames past a sequence's end are NaN in y.

    mass is the same sum over magnitudes. On its way to an output a term takes: two products of up to dk + 64 terms by matrix
    instructions, 2 u each; the roundings of its factors (64 allows for those and for decays from a table); a state's rounding once a
    chunk of 16 frames or more, three operations each. A term passes one value that is held in pieces, its score or the state. With
    16-bit inputs those are two of 8 bits: the first is cut off, which leaves less than 2^-7 of the value's power of two 2^e, below
    2^(e-7), where bf16 has steps of 2^(e-15); the second is rounded to those, off by 2^(e-16) at most: 2^-16. With fp32 inputs
    products of second and third pieces are left out, 2^-7 2^-14 each and two of them."""
    H = log_decay.shape[0]
    B, T = q.shape[:2]
    dk, dv = q.shape[3], v.shape[3]
    q, k, v = heads(q, H), heads(k, H), heads(v, H)
    d = np.exp(np.minimum(log_decay.astype(np.float64), 0.0))[None, :, None, None]
    S = np.zeros((B, H, dk, dv)) if state is None else state.astype(np.float64).copy()
    M = np.abs(S)
    y, mass = np.full((B, T, H, dv), np.nan), np.zeros((B, T, H, dv))
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    for t in range(T):
        on = (t < n)[:, None, None, None]
        kv = k[:, t, :, :, None] * v[:, t, :, None, :]
        S = np.where(on, d * S + kv, S)
        M = np.where(on, d * M + np.abs(kv), M)
        y[:, t] = np.where(on[..., 0], scale * np.einsum("bhd,bhde->bhe", q[:, t], S), np.nan)
        mass[:, t] = abs(scale) * np.einsum("bhd,bhde->bhe", np.abs(q[:, t]), M)
    steps = 64 + 3 * T / 16
    pieces = 2.0 ** -16 if kind != "f32" else 2 * 2.0 ** -21
    # (the outputs' sums and the states' products below 2^-126 may be lost)
    bound = ((dk / 4 + steps) * 2 * U + pieces) * mass + HALF[kind] * np.abs(y) + TINY[kind] + 1e-36
    return y, bound, S, steps * 2 * U * M + 1e-36


def select(logits, scores, n, finished=None, eos=0):
    """(scores float64, parents, tokens), by a sort of all candidates."""
    B, K, V = logits.shape
    best = np.full((B, n), -np.inf)
    parents, tokens = np.zeros((B, n), np.int32), np.full((B, n), eos, np.int32)
    for b in range(B):
        cand = np.full((K, V), -np.inf)
        for k in range(K):
            s = float(scores[b, k])
            if not s > -np.inf:
                continue
            if finished is not None and finished[b, k]:
                cand[k, eos] = s
                continue
            x = logits[b, k].astype(np.float64)
            m = x.max()
            if np.isfinite(m):
                with np.errstate(invalid="ignore"):
                    cand[k] = s + ((x - m) - np.log(np.exp(x - m).sum()))  # (m + log would lose the log beside a mask of -3e38)
        cand = cand.ravel()
        cand[np.isnan(cand)] = -np.inf
        order = np.argsort(-cand, kind="stable")[:n]
        order = order[cand[order] > -np.inf]
        c = len(order)
        best[b, :c], parents[b, :c], tokens[b, :c] = cand[order], order // V, order % V
    return best, parents, tokens


def embedding_grad(g, ids, V, scale):
    """(gradient, bound): the rows of a label are added in fp32, in some order, then scaled."""
    out, mass, count = np.zeros((V, g.shape[1])), np.zeros((V, g.shape[1])), np.zeros(V)
    ok = (ids >= 0) & (ids < V)
    np.add.at(out, ids[ok], g[ok].astype(np.float64))
    np.add.at(mass, ids[ok], np.abs(g[ok].astype(np.float64)))
    np.add.at(count, ids[ok], 1)
    return out * scale, (count[:, None] + 2) * U * mass * abs(scale)
