"""Plain implementations of the paged-serving operators (test infrastructure):
page plans, cache writes and page copies with Python lists, attention and beam
selection in float64, straight from the definitions in include/mtp.h."""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


def plan(length, add, table, num_pages, max_tokens, parent=None):
    """Dict of the arrays that mtp_pages_plan writes."""
    n, m = len(length), table.shape[1]
    rows, status = [], [0, 0, 0, 0]
    for c in range(n):
        p = c if parent is None else int(parent[c])
        ok = 0 <= p < n and add[c] >= 0
        ok = ok and length[p] >= 0 and int(length[p]) + int(add[c]) <= PAGE * m
        rows.append((p, int(length[p]), int(add[c])) if ok else None)
        status[1] += not ok
    kept, used, heads = [], set(), set()
    for row in rows:
        p, L, _ = row or (0, 0, 0)
        keep = L // PAGE
        first = row is not None and p not in heads
        if row is not None:
            heads.add(p)
        if L % PAGE and first:
            keep += 1
        ids = []
        for j in range(keep):
            pg = int(table[p][j])
            if 0 <= pg < num_pages:
                used.add(pg)
            else:
                pg = -1
                status[2] += 1
            ids.append(pg)
        kept.append(ids)
    free = iter([pg for pg in range(num_pages) if pg not in used])
    out = {"table": np.full((n, m), -1, np.int32), "row_start": np.zeros(n + 1, np.int32),
           "kv_len": np.zeros(n, np.int32), "slots": np.full(max_tokens, -1, np.int32),
           "positions": np.full(max_tokens, -1, np.int32), "copies": np.full((n, 2), -1, np.int32)}
    t = 0
    for c, row in enumerate(rows):
        p, L, A = row or (0, 0, 0)
        ids = list(kept[c])
        while len(ids) < -(-(L + A) // PAGE):
            ids.append(next(free, -1))
            status[0] += ids[-1] < 0
        out["table"][c, :len(ids)] = ids
        out["kv_len"][c] = L + A
        if L % PAGE and len(kept[c]) == L // PAGE:
            src, dst = int(table[p][L // PAGE]), ids[L // PAGE]
            if 0 <= src < num_pages and dst >= 0:
                out["copies"][c] = src, dst
        for i in range(A):
            if t < max_tokens:
                pg = ids[(L + i) // PAGE]
                out["slots"][t] = pg * PAGE + (L + i) % PAGE if pg >= 0 else -1
                out["positions"][t] = L + i
            else:
                status[3] += 1
            t += 1
        out["row_start"][c + 1] = t
    out["status"] = np.array(status, np.int32)
    return out


def write(pool, transposed, slots, k, v):
    """pool [pages][2][heads][16 * dim] changed in place; k, v [tokens][heads][dim]."""
    P, _, H, B = pool.shape
    D = B // PAGE
    for t, s in enumerate(slots):
        if not 0 <= s < P * PAGE:
            continue
        pool[s // PAGE, 0].reshape(H, PAGE, D)[:, s % PAGE] = k[t]
        if transposed:
            pool[s // PAGE, 1].reshape(H, D, PAGE)[:, :, s % PAGE] = v[t]
        else:
            pool[s // PAGE, 1].reshape(H, PAGE, D)[:, s % PAGE] = v[t]


def attend(pool, transposed, table, row_start, kv_len, q, out, causal=True, window=0, scale=None, bound=None):
    """out [tokens][heads][dim] float64, changed in place where a row has the token.  bound, of the same shape,
    receives sum_j p_j |V_j| and, in bound_s = bound[1], the largest sum of |scale q_d K_d| over the seen keys."""
    P, _, H, B = pool.shape
    D = B // PAGE
    m = table.shape[1]
    T, HQ, _ = q.shape
    scale = D ** -0.5 if scale is None else scale
    for c in range(len(kv_len)):
        a, b = (min(max(int(x), 0), T) for x in row_start[c:c + 2])
        kv = min(max(int(kv_len[c]), 0), PAGE * m)
        pages = np.array(table[c, :(kv + PAGE - 1) // PAGE], np.int64)
        good = (pages >= 0) & (pages < P)
        raw = pool[np.where(good, pages, 0)].astype(np.float64)                       # [n][2][H][B]
        ks = raw[:, 0].reshape(-1, H, PAGE, D).transpose(0, 2, 1, 3).reshape(-1, H, D)[:kv]
        vs = raw[:, 1].reshape(-1, H, D, PAGE).transpose(0, 3, 1, 2) if transposed else \
            raw[:, 1].reshape(-1, H, PAGE, D).transpose(0, 2, 1, 3)
        vs = vs.reshape(-1, H, D)[:kv]
        j = np.arange(kv)
        there = np.repeat(good, PAGE)[:kv]
        for t in range(a, b):
            pos = kv - (b - a) + (t - a)
            seen = there.copy()
            if causal:
                seen &= j <= pos
                if window > 0:
                    seen &= pos - j < window
            for h in range(HQ):
                out[t, h] = 0.0
                if not seen.any():
                    continue
                x = q[t, h].astype(np.float64)
                k, v = ks[seen, h // (HQ // H)], vs[seen, h // (HQ // H)]
                s = scale * (k @ x)
                w = np.exp(s - (s.max() if s.max() != -np.inf else 0.0))
                w /= w.sum() if w.sum() != 0 else 1.0       # (scores of -infinity only: zeros)
                out[t, h] = w @ v
                if bound is not None:
                    bound[0][t, h] = w @ np.abs(v)
                    bound[1][t, h] = np.abs(scale) * (np.abs(k) @ np.abs(x)).max()
    return out


def beams(logits, score, length, done, eos, eos_min=0, alpha=0.0):
    """(score, length, done, parent, token), each [requests][beams]; logits [requests][beams][vocab]."""
    R, W, V = logits.shape
    out = [np.zeros((R, W), np.float64)] + [np.zeros((R, W), np.int32) for _ in range(4)]
    for r in range(R):
        cand = []
        for b in range(W):
            x = logits[r, b].astype(np.float64)
            if done[r, b]:
                lp = np.full(V, -np.inf)
                lp[eos] = 0.0
                n = int(length[r, b])
            else:
                x = np.where(np.isnan(x), -np.inf, x)
                if length[r, b] < eos_min:
                    x[eos] = -np.inf
                with np.errstate(invalid="ignore", divide="ignore"):
                    lp = x - (x.max() + np.log(np.exp(x - x.max()).sum()))
                n = int(length[r, b]) + 1
            with np.errstate(invalid="ignore"):
                total = np.float64(score[r, b]) + lp
            total = np.where(total < np.inf, total, -np.inf)             # NaN too
            rank = total / max(n, 1) ** float(np.float32(alpha))
            # the best W of the beam are enough: by rank, of equal ones (rounded alike) by logit, then by token
            key = np.zeros(V) if done[r, b] else np.where(np.isfinite(total), x, 0.0)
            for i, v in enumerate(np.lexsort((np.arange(V), -key, -rank))[:W]):
                cand.append((-rank[v], b, i, total[v], n, int(v)))
        cand.sort(key=lambda c: c[:3])
        for i, (_, b, _, s, n, v) in enumerate(cand[:W]):
            out[0][r, i] = s
            out[1][r, i] = n
            out[2][r, i] = int(bool(done[r, b]) or v == eos)
            out[3][r, i] = r * W + b
            out[4][r, i] = v
    return out
