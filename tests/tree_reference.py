"""Plain 64-bit implementations of the calls around trees of drafted tokens (CPU, loops over requests).  Nothing here uses the library."""
import math

import numpy as np

from gqa_reference import PAGE, e4m3

NODES = 64


def masks(parents, text):
    """Of one request: (masks, positions)."""
    if len(parents) > NODES:
        return [0] * len(parents), [-1] * len(parents)
    sets = []
    for t, p in enumerate(parents):
        sets.append((sets[p] if 0 <= p < t else 0) | 1 << t)
    return sets, [text + bin(m).count("1") - 1 for m in sets]


def kept(mask, L, n, sink, window):
    """Cache slots that a query with this mask keeps."""
    nodes = [a for a in range(min(n, NODES)) if mask >> a & 1]
    if not nodes:
        return []
    text, reach = L - n, L - n + len(nodes)
    return ([j for j in range(max(min(text, L), 0)) if j < sink or j >= reach - window]
            + [text + a for rank, a in enumerate(nodes) if text + a >= 0 and (text + rank < sink or text + rank >= reach - window)])


def attend(q, codes_k, codes_v, scales_k, scales_v, page_table, lens, q_start, sets, sink, window, softmax_scale, out_bits, weight_bits):
    """As gqa_reference.attend (errors too), for queries that see what their masks say."""
    tokens, q_heads, dim = q.shape
    heads = codes_k.shape[1]
    group, each = q_heads // heads, PAGE // scales_k.shape[2]
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    out_tol, lse_tol = np.zeros(q.shape), np.zeros(q.shape[:2])
    scale = float(np.float32(softmax_scale))
    for b, L in enumerate(lens):
        n = q_start[b + 1] - q_start[b]
        for t in range(n):
            at = q_start[b] + t
            slots = np.array(kept(sets[at], L, n, sink, window), dtype=np.int64)
            if not slots.size:
                continue
            page, place = np.asarray(page_table[b])[slots // PAGE], slots % PAGE
            for h in range(heads):
                k = codes_k[page, h, place] * scales_k[page, h, place // each][:, None]
                v = codes_v[page, h, place] * scales_v[page, h, place // each][:, None]
                x = q[at, h * group:(h + 1) * group]
                logits = (x @ k.T) * scale
                top = logits.max(1, keepdims=True)
                p = np.exp(logits - top)
                z = p.sum(1, keepdims=True)
                rows = slice(h * group, (h + 1) * group)
                out[at, rows] = (p / z) @ v
                lse[at, rows] = top[:, 0] + np.log(z[:, 0])
                e = 2 * dim * 2.0 ** -24 * abs(scale) * (np.abs(x) @ np.abs(k).T).max(1) + 2.0 ** -20
                lse_tol[at, rows] = e + slots.size * 2.0 ** -24 + 2.0 ** -22 * np.abs(lse[at, rows])
                spread = (p / z) @ np.abs(v)
                out_tol[at, rows] = ((2 * (e[:, None] + 2.0 ** -weight_bits) + slots.size * 2.0 ** -23) * spread
                                     + slots.size * 2.0 ** -35 * np.abs(v).max(0) / z + 2.0 ** -out_bits * np.abs(out[at, rows]))
    return out, lse, out_tol, lse_tol


def attend_bf16(*args):
    # (weights of 22 bits; rounding to bf16 is off by half a step, at most 2^-8 of the number)
    return attend(*args, out_bits=8, weight_bits=22)


def attend_fp32(*args):
    return attend(*args, out_bits=23, weight_bits=22)


def verify(logits, q, tokens, parents, T, uniforms):
    """Of one request: (path, tokens, logprobs).  logits [nodes, vocab] and q (or None) in 64 bits."""
    n, vocab = logits.shape
    if n > NODES:
        return [], [], []
    path, said, chances, at = [], [], [], 0 if n else None
    while at is not None:
        row = np.where(np.isnan(logits[at]), -np.inf, logits[at])
        children = [c for c in range(at + 1, n) if parents[c] == at]
        top = row.max()
        best = int(np.argmax(row))
        if top == -np.inf:
            p = np.zeros(vocab)
        elif top == np.inf:
            p = (np.arange(vocab) == best).astype(float)
        else:
            with np.errstate(over="ignore", invalid="ignore"):
                w = np.exp(np.where(row == -np.inf, -np.inf, (row - top) / (T if T > 0 else 1.0)))
            p = w / w.sum()
        y, go = -1, None
        if top == -np.inf:
            pass
        elif not T > 0:
            y = best
        else:
            weights = p
            if q is not None and children:
                x = tokens[children[0]]
                if 0 <= x < vocab and uniforms[at, 0] * q[at, x] < p[x]:
                    go, y = children[0], x
                else:
                    rest = np.fmax(p - q[at], 0)
                    weights = rest if rest.sum() > 0 else p
            if go is None:
                sums = np.cumsum(weights)
                y = int(np.searchsorted(sums, uniforms[at, 1] * sums[-1], side="right"))
        if go is None and y >= 0:
            go = next((c for c in children if tokens[c] == y), None)
        path.append(at)
        said.append(y)
        chances.append(0.0 if y < 0 else math.log(p[y]) if p[y] > 0 else -math.inf)
        at = go
    return path, said, chances


def keep(path, lens, q_start, page_table, codes, scales):
    """codes (their values) [layers, pages, heads, 128, dim] and scales [layers, pages, heads, blocks] in 64 bits (scales of 32), changed in place."""
    each = PAGE // scales.shape[3]
    for b, L in enumerate(lens):
        n = q_start[b + 1] - q_start[b]
        text, way = L - n, []
        if n > NODES or text < 0:
            continue
        for i, p in enumerate(path[q_start[b]:q_start[b + 1]]):
            if not (i <= p < n and (i == 0 or p > way[-1])):
                break
            way.append(p)

        def slot(at):
            return page_table[b][at // PAGE], at % PAGE
        rows = [(codes[:, slot(text + p)[0], :, slot(text + p)[1]].copy(), scales[:, slot(text + p)[0], :, slot(text + p)[1] // each].copy()) for p in way]
        for block in sorted({(text + i) // each for i, p in enumerate(way) if p != i}):
            page, low = slot(block * each)
            mine = [i for i in range(len(way)) if (text + i) // each == block]
            held = max(0, text - block * each)
            old = scales[:, page, :, low // each].copy()
            new = np.max([rows[i][1] for i in mine] + ([old] if held else []), axis=0)

            def recoded(values, was):
                ratio = np.where(new > 0, np.float32(was) / np.where(new > 0, new, 1).astype(np.float32), np.float32(1)).astype(np.float64)
                while ratio.ndim < values.ndim:
                    ratio = ratio[..., None]
                with np.errstate(invalid="ignore"):
                    return np.where(ratio == 1, values, e4m3((values * ratio).astype(np.float32).astype(np.float64)))
            codes[:, page, :, low:low + held] = recoded(codes[:, page, :, low:low + held], old)
            for i in mine:
                codes[:, page, :, slot(text + i)[1]] = recoded(*rows[i])
            scales[:, page, :, low // each] = new


def truncate(lens, dropped, page_table, stack, count, entries):
    """(lens, stack, count)."""
    lens, stack = list(lens), list(stack)
    for b, (L, d) in enumerate(zip(lens, dropped)):
        left = L - min(max(d, 0), max(L, 0))
        for page in page_table[b][-(-max(left, 0) // PAGE):-(-max(L, 0) // PAGE)]:
            if count < entries:
                stack[count] = page
                count += 1
        lens[b] = left
    return lens, stack, count
