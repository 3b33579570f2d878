"""Independent oracle of the rollout operators: numpy in 64 bits, element by element where that is clearest, from the
definitions alone.  Test infrastructure only; shares no code with the library.

Every function also returns what its caller derives tolerances from (sums of absolute values)."""
import numpy as np


def rotate(x, positions, cos, sin, interleaved):
    """x [token, head, element] turned pair by pair; returns (turned, |a| + |b| of every element's pair)."""
    x = x.astype(np.float64)
    out, size = x.copy(), np.zeros_like(x)
    pairs = cos.shape[1]
    for i in range(pairs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        c, s = (t[positions, i].astype(np.float64)[:, None] for t in (cos, sin))
        out[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        out[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
        size[:, :, a] = size[:, :, b] = np.abs(x[:, :, a]) + np.abs(x[:, :, b])
    return out, size


def visible(pages, length, table_row, page_tokens, n_pages, bound):
    """[(page, token of the page)] of the visible tokens of one table row."""
    length = max(0, min(int(length), bound, len(table_row) * page_tokens))
    places = []
    for t in range(length):
        page = int(table_row[t // page_tokens])
        if 0 <= page < n_pages:
            places.append((page, t % page_tokens))
    return places


def attend(q, k, v, suffix_lens, suffix_pages, group_offsets, prefix_lens, prefix_pages, scale, max_group=None, max_prefix=None, max_suffix=None):
    """q [sequence, query head, element]; k, v [page, KV head, token, element].  Returns out, lse, and for tolerances
    sum p |v| and the largest sum |q| |k| * |scale| of every row."""
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    n, hq, d = q.shape
    n_pages, hk, page_tokens, _ = k.shape
    out, size = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, score = np.full((n, hq), -np.inf), np.zeros((n, hq))
    big = 1 << 40
    for i in range(n):
        places = []
        if group_offsets is not None:
            for g in range(len(prefix_lens)):
                at = i - int(group_offsets[g])
                if 0 <= at < int(group_offsets[g + 1]) - int(group_offsets[g]) and (max_group is None or at < max_group):
                    places += visible(k, prefix_lens[g], prefix_pages[g], page_tokens, n_pages, big if max_prefix is None else max_prefix)
        places += visible(k, suffix_lens[i], suffix_pages[i], page_tokens, n_pages, big if max_suffix is None else max_suffix)
        if not places:
            continue
        at = tuple(np.array(p) for p in zip(*places))
        for h in range(hq):
            kv = h // (hq // hk)
            keys, values = k[at[0], kv, at[1]], v[at[0], kv, at[1]]
            x = scale * (keys @ q[i, h])
            score[i, h] = abs(scale) * (np.abs(keys) @ np.abs(q[i, h])).max()
            m = x.max()
            e = np.exp(x - m)
            lse[i, h] = m + np.log(e.sum())
            p = e / e.sum()
            out[i, h], size[i, h] = p @ values, p @ np.abs(values)
    return out, lse, size, score


def logprobs(x, targets, temperature):
    """Log probabilities of the targets, entropy and lse of rows of logits; a row whose target is outside the vocabulary is all
    zeros (no targets: every row counts).  Also log p of every element."""
    with np.errstate(all="ignore"):
        y = x.astype(np.float64) / temperature
        rows, vocab = y.shape
        top = y.max(1, keepdims=True)
        base = np.where(top == -np.inf, 0.0, top)
        z = np.exp(y - base).sum(1, keepdims=True)
        lse = base + np.log(z)
        logp = np.where(y == -np.inf, -np.inf, y - base - np.log(z))
        p = np.exp(logp)
        ent = -np.where(p == 0, 0.0, p * logp).sum(1)
    live = np.ones(rows, bool) if targets is None else (targets >= 0) & (targets < vocab)
    given = np.where(live, 0 if targets is None else targets, 0)
    lp = logp[np.arange(rows), given]
    return np.where(live, lp, 0.0), np.where(live, ent, 0.0), np.where(live, lse[:, 0], 0.0), logp, live


def top_ids(x, n):
    """The n largest of every row, larger first, equal ones (0 and -0 among them) by the lower index."""
    return np.stack([np.lexsort((np.arange(x.shape[1]), -row.astype(np.float64)))[:n] for row in x])


def logprobs_back(x, targets, temperature, grad_logprob, grad_entropy):
    lp, ent, lse, logp, live = logprobs(x, targets, temperature)
    p = np.exp(logp)
    hot = np.zeros(x.shape)
    hot[np.arange(len(x))[live], targets[live]] = 1
    g, h = grad_logprob[:, None], grad_entropy[:, None]
    with np.errstate(all="ignore"):
        dx = (g * (hot - p) - h * np.where(p == 0, 0.0, p * (logp + ent[:, None]))) / temperature
    return np.where(live[:, None], dx, 0.0), p, logp
