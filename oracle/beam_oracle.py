"""fp64 CPU oracle of beam search: selection over beams and vocabulary, and the
reordering of the beams' states.

TEST INFRASTRUCTURE ONLY, as ``aal_oracle``: a plain transcription of the
definitions in ``include/aal.h``, sharing no code with the HIP library.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["select", "reorder"]


def select(z, scores, n, T=1.0, finished=None, lengths=None, alpha=0.0, eos=-1, pad=0):
    """Dict of [B, n] arrays: scores, rank, parents, tokens, finished, lengths."""
    z, scores = np.asarray(z, np.float64), np.asarray(scores, np.float64)
    B, W, V = z.shape
    out = {"scores": np.full((B, n), -math.inf), "rank": np.full((B, n), -math.inf), "parents": np.full((B, n), -1),
           "tokens": np.full((B, n), pad), "finished": np.ones((B, n), bool), "lengths": np.zeros((B, n), int)}
    for b in range(B):
        cands = []  # (-rank, beam, -logit, token, total, ended, length)
        for w in range(W):
            if scores[b, w] == -math.inf:
                continue
            length = 0 if lengths is None else int(lengths[b, w])
            if finished is not None and finished[b, w]:
                rank = scores[b, w] / length ** alpha if alpha else scores[b, w]
                cands.append((-rank, w, 0.0, pad, scores[b, w], True, length))
                continue
            x = z[b, w] / T
            m = x.max()
            if m == -math.inf:
                continue
            total = scores[b, w] + (x - (m + np.log(np.exp(x - m).sum())))
            rank = total / (length + 1) ** alpha if alpha else total
            for v in np.lexsort((np.arange(V), -(z[b, w] + 0.0)))[:n]:
                if z[b, w, v] > -math.inf:
                    cands.append((-rank[v], w, -(z[b, w, v] + 0.0), int(v), total[v], int(v) == eos, length + 1))
        for j, c in enumerate(sorted(cands)[:n]):
            out["rank"][b, j], out["parents"][b, j], out["tokens"][b, j] = -c[0], c[1], c[3]
            out["scores"][b, j], out["finished"][b, j], out["lengths"][b, j] = c[4], c[5], c[6]
    return out


def reorder(state, parents, before=None):
    """state [B, W, ...] by parents [B, n]; a slot without a parent keeps what `before` (the state) has."""
    state, parents = np.asarray(state), np.asarray(parents)
    out = (state if before is None else np.asarray(before)).copy()
    for b in range(parents.shape[0]):
        for j in range(parents.shape[1]):
            if 0 <= parents[b, j] < state.shape[1]:
                out[b, j] = state[b, parents[b, j]]
    return out
