"""Independent oracle of what surrounds a rollout's steps: numpy in 64 bits and plain Python, row by row, from the
definitions alone.  Test infrastructure only; shares no code with the library.

The numerical functions also return what their callers derive tolerances from (sums of absolute values)."""
import numpy as np


def adjust(x, tokens=None, lens=None, prompt_lens=None, repetition=None, frequency=None, presence=None, bias_ids=None, bias=None, allowed=None,
           allowed_rows=None):
    """Adjusted logits, which of them anything applied to, and the sum of the absolute values that went into each."""
    rows, vocab = x.shape
    out, size, touched = x.astype(np.float64), np.abs(x.astype(np.float64)), np.zeros((rows, vocab), bool)
    with np.errstate(all="ignore"):
        for r in range(rows):
            seen, answer = {}, {}
            n = 0 if tokens is None else max(0, min(int(lens[r]), tokens.shape[1]))
            for i in range(n):
                t = int(tokens[r, i])
                if 0 <= t < vocab:
                    seen[t] = True
                    if prompt_lens is None or i >= prompt_lens[r]:
                        answer[t] = answer.get(t, 0) + 1
            f, p, rep = (float(d if a is None else a[r]) for a, d in ((frequency, 0), (presence, 0), (repetition, 1)))
            for t in seen:
                v = out[r, t]
                v = v / rep if v > 0 else v * rep
                out[r, t], size[r, t], touched[r, t] = v, abs(v), True
                if t in answer:
                    out[r, t] = v - f * answer[t] - p
                    size[r, t] += abs(f) * answer[t] + abs(p)
            given = {} if bias is None else {int(t): float(b) for t, b in zip(bias_ids[r], bias[r]) if 0 <= t < vocab}
            for t, b in given.items():
                out[r, t] += b
                size[r, t] += abs(b)
                touched[r, t] = True
            if allowed is not None:
                g = r if allowed_rows is None else int(allowed_rows[r])
                if 0 <= g < len(allowed):
                    for t in range(vocab):
                        if not int(allowed[g, t // 32]) >> (t % 32) & 1:
                            out[r, t], touched[r, t] = -np.inf, True
    return out, touched, size


def distill(x, ids, logprobs, temperature, reverse, rest):
    """Loss of every row and its gradient; for tolerances the sizes of what the loss and the gradients are made of, and -log of every probability (0 where p = 0)."""
    rows, vocab = x.shape
    loss, grad = np.zeros(rows), np.zeros((rows, vocab))
    loss_size, grad_size, spread = np.zeros(rows), np.zeros((rows, vocab)), np.zeros((rows, vocab))
    w = float(reverse)
    live = np.zeros(rows, bool)
    with np.errstate(all="ignore"):
        for r in range(rows):
            named = {}
            for t, l in zip(ids[r], logprobs[r]):
                if 0 <= t < vocab and l != -np.inf:
                    named.setdefault(int(t), float(l))
            if not named:
                continue
            live[r] = True
            y = x[r].astype(np.float64) / temperature
            top = y.max()
            e = np.exp(y - (0 if top == -np.inf else top))
            z = e.sum()
            logp = np.where(y == -np.inf, -np.inf, y - (0 if top == -np.inf else top) - np.log(z))
            other = np.ones(vocab, bool)
            other[list(named)] = False
            z_other = e[other].sum()
            # (label, q, ln q as the way ahead has it, ln q as the way back has it, p, ln p)
            at = [(t, np.exp(l), l, l, np.exp(logp[t]), logp[t]) for t, l in named.items()]
            q_sum = sum(a[1] for a in at)
            if rest and not z_other <= 0:
                q = max(0.0, 1 - q_sum)
                # its logarithm from its own largest element: the sum itself may be too small for 64 bits
                y_other = y[other].max()
                lp = y_other + np.log(np.exp(y[other] - y_other).sum()) - top - np.log(z)
                at.append((None, q, np.log(q) if q > 0 else 0.0, np.log(max(1 - q_sum, 2.0 ** -24)), np.exp(lp), lp))
            ahead = [0.0 if q == 0 else q * (lq - lp) for _, q, lq, _, p, lp in at]
            back = [0.0 if p == 0 else p * (lp - lq) for _, q, _, lq, p, lp in at]
            loss[r] = (0.0 if w == 1 else (1 - w) * sum(ahead)) + (0.0 if w == 0 else w * sum(back))
            loss_size[r] = (1 - w) * sum(q for _, q, *_ in at) + w * sum(0.0 if p == 0 else p * (abs(lp - lq) + 1) for _, q, _, lq, p, lp in at)
            # d loss / d p of each, times p, then through the softmax: p_i (f_i - sum f p)
            fp = {}
            for t, q, _, lq, p, lp in at:
                fp[t] = (0.0 if w == 1 else -(1 - w) * q) + (0.0 if w == 0 or p == 0 else w * p * (lp - lq + 1))
            total = sum(fp.values())
            size_of = {t: (1 - w) * (q + p) + (0.0 if p == 0 else w * p * (abs(lp - lq) + 2 + abs(sum(back)))) for t, q, _, lq, p, lp in at}
            share = np.zeros(vocab)
            if z_other > 0:
                share = np.where(other & (y > -np.inf), np.exp(y - y[other].max() - np.log(np.exp(y[other] - y[other].max()).sum())), 0.0)
            p_other = np.exp(logp[other]).sum()
            grad[r] = share * ((fp.get(None, 0.0)) - p_other * total) / temperature
            grad_size[r] = share * (size_of.get(None, p_other * (1 + abs(total)))) / temperature
            for t, q, _, lq, p, lp in at:
                if t is not None:
                    grad[r, t] = (fp[t] - p * total) / temperature
                    grad_size[r, t] = size_of[t] / temperature
            if np.isnan(x[r]).any() or (x[r] == np.inf).any() or any(np.isnan(l) for l in named.values()):
                loss[r], grad[r] = np.nan, np.nan
            spread[r] = np.where(np.isfinite(y), top - y, 0.0)
    return loss, grad, loss_size, grad_size, spread, live


# ---- pages: books kept as a program on the host would keep them ------------------------------------------------------------

def _rows(tables, lens, page, pages):
    """(length, page numbers) of every row: those of its length, -1 where a number names no page."""
    out = []
    for t, n in zip(tables, lens):
        n = max(0, min(int(n), len(t) * page))
        out.append((n, [int(p) if 0 <= p < pages else -1 for p in t[:-(-n // page)]]))
    return out


def fork(tables, lens, parents, refs, page):
    """(tables, lens, refs, [(source page, new page, tokens)])."""
    pages, width = len(refs), tables.shape[1]
    refs = [int(n) for n in refs]
    old = _rows(tables, lens, page, pages)
    for _, row in old:
        for p in row:
            if p >= 0:
                refs[p] -= 1
    new, taken, wants = [], set(), []
    for r, parent in enumerate(parents):
        n, row = old[parent] if 0 <= parent < len(old) else (0, [])
        row = list(row)
        if n % page and row[-1] >= 0:
            if row[-1] in taken:
                wants.append(r)
            taken.add(row[-1])
        new.append([n, row])
        for i, p in enumerate(row):
            if p >= 0 and not (r in wants and i == len(row) - 1):
                refs[p] += 1
    free = [p for p in range(pages) if refs[p] == 0 and p not in taken]  # (where counts are wrong, one that a row goes on in might have 0)
    copies = []
    for k, r in enumerate(wants):
        n, row = new[r]
        if k < len(free):
            copies.append((row[-1], free[k], n % page))
            row[-1] = free[k]
            refs[free[k]] = 1
        else:
            for p in row[:-1]:
                if p >= 0:
                    refs[p] -= 1
            new[r] = [0, []]
    table = np.array([row + [-1] * (width - len(row)) for _, row in new], np.int32).reshape(len(new), width)
    return table, np.array([n for n, _ in new], np.int32), np.array(refs, np.int32), copies


def grow(tables, lens, counts, refs, most, page):
    """(tables, lens, slots, refs)."""
    pages, width = len(refs), tables.shape[1]
    refs = [int(n) for n in refs]
    free = [p for p in range(pages) if refs[p] == 0]
    used, short = 0, False
    table, ends, slots = [], [], []
    for (n, row), count in zip(_rows(tables, lens, page, pages), counts):
        count = max(0, min(int(count), most))
        want = -(-(n + count) // page)
        need = want - len(row)
        places = [-1] * most
        if want <= width and (need == 0 or not short):
            if used + need <= len(free):
                for p in free[used:used + need]:
                    refs[p] = 1
                    row = row + [p]
                used += need
                for i in range(count):
                    p = row[(n + i) // page]
                    places[i] = p * page + (n + i) % page if p >= 0 else -1
                n += count
            else:
                short = True
        table.append(row + [-1] * (width - len(row)))
        ends.append(n)
        slots.append(places)
    return (np.array(table, np.int32).reshape(len(table), width), np.array(ends, np.int32), np.array(slots, np.int64).reshape(len(slots), most),
            np.array(refs, np.int32))


def compact(refs, tables):
    """(tables, refs, places, n, [(from, to)])."""
    live = [p for p in range(len(refs)) if refs[p]]
    n = len(live)
    room = iter([p for p in range(n) if not refs[p]])
    places = np.full(len(refs), -1, np.int32)
    moves = []
    for p in live:
        places[p] = p if p < n else next(room)
        if p >= n:
            moves.append((p, int(places[p])))
    out = np.zeros(len(refs), np.int32)
    out[places[live]] = np.asarray(refs)[live]
    new = [np.where((t >= 0) & (t < len(refs)), places[np.clip(t, 0, len(refs) - 1)], t) for t in tables]
    return new, out, places, n, moves
