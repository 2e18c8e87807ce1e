"""Plain float64 statement of the operators for several requests behind one shared prefix, and of
the scores of logits rows.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Everything is written request by request and
row by row: lists of pages, explicit key lists, one softmax per row.  Nothing is split, merged or
masked with large numbers.
"""

import math

import numpy as np

PAGE = 64
MAX_ROWS = 128

OK, BAD_LENGTHS, NO_PAGES, BAD_TREE = 0, 1, 2, 3


def plan(row_start, held, parent, prefix_len, block_table, free_pages, n_pages, n_rows, head_dim, theta):
    """One step's plan: dict with block_table (a new one), slot, position, ancestors (a list of rows of the
    request per row, empty for rows of no placed request), rope [n_rows, head_dim / 2, 2], status, taken."""
    B = len(held)
    table = np.array(block_table, dtype=np.int64, copy=True)
    slot, pos = [-1] * n_rows, [0] * n_rows
    anc = [[] for _ in range(n_rows)]
    status, taken = [OK] * B, 0
    count = [row_start[b + 1] - row_start[b] for b in range(B)]
    if row_start[0] != 0 or row_start[B] > n_rows or min(count) < 0 or max(count) > MAX_ROWS or min(held) < 0:
        status = [BAD_LENGTHS] * B
    else:
        for b in range(B):
            end = held[b] + count[b]
            have, want = -(-held[b] // PAGE), -(-end // PAGE)
            mine = range(taken, taken + want - have)
            taken += want - have
            if count[b] == 0:
                continue
            if want > table.shape[1] or taken > len(free_pages) or prefix_len + end > 2**31:
                status[b] = NO_PAGES
                continue
            pages = list(table[b, :have]) + [free_pages[i] for i in mine]
            if any(not 0 <= p < n_pages for p in pages[held[b] // PAGE:]):
                status[b] = NO_PAGES
                continue
            r0 = row_start[b]
            par = list(range(-1, count[b] - 1)) if parent is None else [int(p) for p in parent[r0:r0 + count[b]]]
            if par[0] != -1 or any(not 0 <= par[i] < i for i in range(1, count[b])):
                status[b] = BAD_TREE
                continue
            table[b, :want] = pages
            for i in range(count[b]):
                chain, j = [], i
                while j >= 0:
                    chain.append(j)
                    j = par[j]
                at = held[b] + i
                slot[r0 + i] = pages[at // PAGE] * PAGE + at % PAGE
                pos[r0 + i] = prefix_len + held[b] + len(chain) - 1
                anc[r0 + i] = sorted(chain)
    half = head_dim // 2
    freq = np.array([theta ** (-2.0 * j / head_dim) for j in range(half)])
    ang = np.array(pos, dtype=np.float64)[:, None] * freq
    return {"block_table": table, "slot": np.array(slot), "position": np.array(pos), "ancestors": anc,
            "rope": np.stack([np.cos(ang), np.sin(ang)], -1), "status": np.array(status), "taken": taken}


def mask_words(ancestors):
    """The ancestor lists as four 32-bit words per row."""
    out = np.zeros((len(ancestors), 4), dtype=np.uint32)
    for i, a in enumerate(ancestors):
        for j in a:
            out[i, j // 32] |= np.uint32(1 << (j % 32))
    return out


def turn(x, rope):
    """Rotate-half rotary embedding of x [N, heads, Dh] by a table [N, Dh / 2, 2]."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = rope[:, None, :, 0], rope[:, None, :, 1]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def attention(q, prefix_k, prefix_v, page_k, page_v, block_table, row_start, held, ancestors, n_pages):
    """out [N, H, Dh] and the same sums over the values' sizes (what roundings of the probabilities can
    change): q [N, H, Dh], prefix_k / prefix_v [Hkv, P, Dh], page_k / page_v [n_pages, Hkv, 64, Dh].  Rows of
    no request are NaN."""
    N, H, Dh = q.shape
    Hkv = prefix_k.shape[0]
    out, size = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    for b in range(len(held)):
        for r in range(row_start[b], row_start[b + 1]):
            slots = list(range(held[b])) + [held[b] + j for j in ancestors[r]]
            slots = [t for t in slots if t // PAGE < block_table.shape[1] and 0 <= block_table[b, t // PAGE] < n_pages]
            pages = np.array([block_table[b, t // PAGE] for t in slots], dtype=np.int64)
            offs = np.array([t % PAGE for t in slots], dtype=np.int64)
            for h in range(H):
                kh = h // (H // Hkv)
                k = np.concatenate([prefix_k[kh], page_k[pages, kh, offs]])
                v = np.concatenate([prefix_v[kh], page_v[pages, kh, offs]])
                if len(k) == 0:
                    out[r, h] = size[r, h] = 0.0
                    continue
                z = k @ q[r, h] / math.sqrt(Dh)
                w = np.exp(z - z.max())
                w /= w.sum()
                out[r, h], size[r, h] = w @ v, w @ np.abs(v)
    return out, size


def commit(row_start, slots, path, accept_len, k_rows, v_rows):
    """Moves accepted rows to the front: k_rows / v_rows [L, n_slots, ...] by slot (new arrays)."""
    k, v = k_rows.copy(), v_rows.copy()
    for b in range(len(accept_len)):
        r0, n = row_start[b], row_start[b + 1] - row_start[b]
        if not 1 <= accept_len[b] < n:
            continue
        for i in range(1, accept_len[b] + 1):
            p = path[r0 + i]
            if i < p < n and slots[r0 + p] >= 0:
                k[:, slots[r0 + i]] = k_rows[:, slots[r0 + p]]
                v[:, slots[r0 + i]] = v_rows[:, slots[r0 + p]]
    return k, v


def token_scores(logits, tokens, row_of, k):
    """Scores of float64 logits [n, V] (see the operator's conventions for -inf, NaN and absent tokens)."""
    n, V = logits.shape
    lse, entropy, shift = np.zeros(n), np.zeros(n), np.full((n, 2), np.nan)
    top, top_lp = np.full((n, k), -1), np.full((n, k), -np.inf)
    for r in range(n):
        x = logits[r]
        if np.any(np.isnan(x)) or np.any(x == np.inf):
            lse[r] = entropy[r] = np.nan
            top_lp[r] = np.nan
            continue
        live = np.flatnonzero(x > -np.inf)
        if len(live) == 0:
            lse[r] = -np.inf
            continue
        # (log p = (x - m) - log sum exp(x - m): x - lse loses the logarithm beside an m of 1e38)
        m = x[live].max()
        log_sum = math.log(np.exp(x[live] - m).sum())
        lse[r] = m + log_sum
        shift[r] = m, log_sum
        lp = (x[live] - m) - log_sum
        entropy[r] = -(np.exp(lp) * lp).sum()
        best = live[np.argsort(-x[live], kind="stable")][:k]
        top[r, :len(best)] = best
        top_lp[r, :len(best)] = (x[best] - m) - log_sum
    logprob = np.zeros(len(tokens))
    for i, t in enumerate(tokens):
        r = i if row_of is None else row_of[i]
        if not 0 <= r < n:
            logprob[i] = np.nan
        elif t >= V:
            logprob[i] = np.nan
        elif t >= 0:
            logprob[i] = -np.inf if lse[r] == -np.inf else (logits[r, t] - shift[r, 0]) - shift[r, 1]
    return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_token": top, "top_logprob": top_lp}
