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


def norm(x, gain, eps):
    """RMSNorm of every head of x [N, heads, Dh] with gain [Dh] or [heads, Dh] (None: ones)."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if gain is None else y * gain


def adjust(logits, row_start, held, ancestors, tokens, history=None, prompt_len=None, seen=(), penalties=None, bias=None,
           allow=None, mask_of=None):
    """Adjusted logits of every placed row, one token after the other, each step rounded to fp32 as the operator
    states it: logits float32 [N, V], history a list of token lists, seen a collection of tokens, penalties float32
    [B, 3], bias a list of (token, value) lists, allow a list of sets.  Rows of no placed request are as they were."""
    N, V = logits.shape
    out = logits.astype(np.float32).copy()
    f = np.float32
    for b in range(len(held)):
        for r in range(row_start[b], row_start[b + 1]):
            if not ancestors[r]:
                continue
            text = list(history[b][:held[b]]) if history is not None else []
            text += [None] * (held[b] - len(text))  # (tokens past the history count as absent)
            text += [tokens[row_start[b] + j] for j in ancestors[r]] if tokens is not None else []
            x = out[r]
            if penalties is not None:
                rho, presence, frequency = (f(v) for v in penalties[b])
                answer = {}
                for t in text[prompt_len[b] if prompt_len is not None else 0:]:
                    answer[t] = answer.get(t, 0) + 1
                for t in set(text) | set(seen):
                    if t is None or not 0 <= t < V:
                        continue
                    c = answer.get(t, 0)
                    with np.errstate(all="ignore"):
                        x[t] = f(x[t] / rho) if x[t] > 0 else f(x[t] * rho)
                        x[t] = f(x[t] - f(frequency * f(c)))
                        if c:
                            x[t] = f(x[t] - presence)
            if bias is not None:
                for t, v in dict(bias[b]).items():  # (the last of a token's entries)
                    if 0 <= t < V:
                        with np.errstate(all="ignore"):
                            x[t] = f(x[t] + f(v))
            if allow is not None and mask_of[r] >= 0:
                ok = allow[mask_of[r]] if mask_of[r] < len(allow) else ()
                for t in range(V):
                    if t not in ok:
                        x[t] = -np.inf
    return out


def greedy(row):
    """The token of the largest value, the lowest among equals; -1 if there is none or a NaN."""
    if np.isnan(row).any() or row.max() == -np.inf:
        return -1
    return int(np.flatnonzero(row == row.max())[0])


def accept(tokens, parent, best):
    """One request's walk: (path, token after it).  tokens, parent and best are its rows'."""
    reached = [0]
    depth = [0] * len(tokens)
    for i in range(1, len(tokens)):
        depth[i] = depth[parent[i]] + 1
        if parent[i] in reached and best[parent[i]] >= 0 and tokens[i] == best[parent[i]]:
            reached.append(i)
    end = max(reached, key=lambda i: (depth[i], -i))
    path = []
    i = end
    while i >= 0:
        path.append(i)
        i = parent[i]
    return path[::-1], int(best[end])


def fork(table, held, source, n_pages):
    """What requests that continue from others hold: dict with block_table, held, free, status, and copies, a list of
    (page, new page, tokens).  Requests' pages are lists; who shares a page with whom follows from the order."""
    B, width = table.shape
    old = dict(block_table=table.copy(), held=list(held), free=[], copies=[])
    if any(h < 0 or -(-h // PAGE) > width for h in held) or any(s >= B for s in source):
        return dict(old, status=BAD_LENGTHS)
    mine = [list(table[b, :-(-held[b] // PAGE)]) for b in range(B)]
    taken = {p for pages in mine for p in pages}
    free = [p for p in range(n_pages) if p not in taken]
    owner = {}  # who goes on with a request's last page
    for b, s in enumerate(source):
        if s >= 0 and (s == b or s not in owner):
            owner[s] = b
    pages, copies = [], []
    for b, s in enumerate(source):
        now = list(mine[s]) if s >= 0 else []
        if s >= 0 and owner[s] != b and held[s] % PAGE and 0 <= now[-1] < n_pages:
            copies.append([now[-1], None, held[s] % PAGE])
            now[-1] = copies[-1]
        pages.append(now)
    if len(copies) > len(free):
        return dict(old, status=NO_PAGES)
    for c, p in zip(copies, free):
        c[1] = p
    out = np.full((B, width), -1)
    for b, now in enumerate(pages):
        out[b, :len(now)] = [p[1] if isinstance(p, list) else p for p in now]
    left = set(out.reshape(-1).tolist())
    return dict(block_table=out, held=[held[s] if s >= 0 else 0 for s in source], status=OK,
                free=[p for p in range(n_pages) if p not in left], copies=[tuple(c) for c in copies])


def compact(table, held, n_pages):
    """(new table, pages in use, moves as (page, new page))."""
    B, width = table.shape
    mine = [[p for p in table[b, :min(-(-max(held[b], 0) // PAGE), width)]] for b in range(B)]
    used = sorted({p for pages in mine for p in pages if 0 <= p < n_pages})
    holes = [p for p in range(len(used)) if p not in set(used)]
    moves = list(zip([p for p in used if p >= len(used)], holes))
    to = dict(moves)
    out = np.full((B, width), -1)
    for b, pages in enumerate(mine):
        out[b, :len(pages)] = [to.get(p, p) if 0 <= p < n_pages else -1 for p in pages]
    return out, len(used), moves
