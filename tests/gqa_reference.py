"""Plain 64-bit implementations of the grouped-query calls (CPU, loops over requests), and the error bounds that the
kernels' arithmetic allows.  Nothing here uses the library."""
import math

import numpy as np
import torch

PAGE = 128


def extend(seq_lens, new_lens, free_pages, free_count, page_table, max_tokens):
    """Lists in, lists out: (page_table, seq_lens, free_count, q_start, slot_map)."""
    table = [list(r) for r in page_table]
    lens, q_start, slots = list(seq_lens), [0], [-1] * max_tokens
    lacked = taken = 0
    for b, (L, n) in enumerate(zip(seq_lens, new_lens)):
        begin = q_start[-1]
        q_start.append(min(begin + max(n, 0), 2 ** 31 - 1))   # (int32: the sums stop there)
        if L < 0 or n < 0 or -(-(L + n) // PAGE) > len(table[b]) or begin + n > max_tokens:
            continue
        had, has = -(-L // PAGE), -(-(L + n) // PAGE)
        first = lacked
        lacked += has - had
        if has > had and lacked > free_count:
            continue
        for k in range(has - had):
            table[b][had + k] = free_pages[free_count - 1 - first - k]
        if has > had:
            taken = lacked
        for t in range(n):
            slots[begin + t] = table[b][(L + t) // PAGE] * PAGE + (L + t) % PAGE
        lens[b] = L + n
    return table, lens, free_count - taken, q_start, slots


def e4m3(x):
    """Numbers of magnitude up to 448 (64 bits) to the nearest that e4m3 holds, ties to even; others to NaN."""
    exponent = np.maximum(np.floor(np.log2(np.maximum(np.abs(np.nan_to_num(x)), 2.0 ** -30))), -6)
    step = 2.0 ** (exponent - 3)
    with np.errstate(invalid="ignore"):
        y = np.rint(x / step) * step
        return np.where(np.abs(y) <= 448, y, np.nan)


def append(new, slots, codes, scales):
    """new [tokens, heads, dim]; codes (values of the codes) [pages, heads, 128, dim] and scales [pages, heads, blocks] in 64 bits, changed
    in place.  Returns which tokens' values are defined afterwards, [pages, heads, 128] (those behind the last written in a block are not)."""
    each = PAGE // scales.shape[2]
    defined = np.ones(codes.shape[:3], dtype=bool)
    runs, i = [], 0
    while i < len(slots):
        j = i + 1
        while j < len(slots) and slots[j] == slots[i] + (j - i) and slots[j] // each == slots[i] // each:
            j += 1
        if 0 <= slots[i] < codes.shape[0] * PAGE:
            runs.append((i, j))
        i = j
    for i, j in runs:
        page, place = divmod(int(slots[i]), PAGE)
        block, low = place // each, place % each
        for h in range(codes.shape[1]):
            x = new[i:j, h]
            finite = np.abs(x[np.isfinite(x)])
            top = finite.max() if finite.size else 0.0
            scale = 0.0
            if top > 0:
                scale = 2.0 ** max(-126, math.ceil(math.log2(top / 448)))
            if low:
                old = scales[page, h, block]
                scale = max(scale, old)
                if scale > old:
                    held = codes[page, h, block * each:place]
                    codes[page, h, block * each:place] = e4m3(held * (old / scale))
            y = np.where(np.isfinite(x), x / scale if scale > 0 else 0.0, np.nan)
            codes[page, h, place:place + (j - i)] = e4m3(y)
            scales[page, h, block] = scale
            defined[page, h, place + (j - i):(block + 1) * each] = False
    return defined


def attend(q, codes_k, codes_v, scales_k, scales_v, page_table, seq_lens, q_start, sink, window, softmax_scale, out_bits, weight_bits):
    """q [tokens, query heads, dim] and the cache in 64 bits.  Returns out, lse, and the largest errors that the kernel's arithmetic allows
    for each: logits are sums of dim products in 32 bits, weights carry weight_bits significant bits (and at least 2^-35 of the
    largest one), sums run over the kept tokens in 32 bits, the result is rounded to out_bits."""
    tokens, q_heads, dim = q.shape
    heads = codes_k.shape[1]
    group, each = q_heads // heads, PAGE // scales_k.shape[2]
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    out_tol, lse_tol = np.zeros(q.shape), np.zeros(q.shape[:2])
    scale = float(np.float32(softmax_scale))
    for b, L in enumerate(seq_lens):
        n = q_start[b + 1] - q_start[b]
        for t in range(n):
            reach = L - n + t + 1
            kept = np.array([j for j in range(max(reach, 0)) if j < sink or j >= reach - window], dtype=np.int64)
            if not kept.size:
                continue
            page, place = np.asarray(page_table[b])[kept // PAGE], kept % PAGE
            for h in range(heads):
                k = codes_k[page, h, place] * scales_k[page, h, place // each][:, None]
                v = codes_v[page, h, place] * scales_v[page, h, place // each][:, None]
                for g in range(group):
                    x = q[q_start[b] + t, h * group + g]
                    logits = (k @ x) * scale
                    top = logits.max()
                    p = np.exp(logits - top)
                    z = p.sum()
                    at = (q_start[b] + t, h * group + g)
                    out[at] = (p / z) @ v
                    lse[at] = top + math.log(z)
                    # (a factor of two for the roundings of the factors and of exp2, which are smaller)
                    e = 2 * dim * 2.0 ** -24 * abs(scale) * (np.abs(k) @ np.abs(x)).max() + 2.0 ** -20
                    lse_tol[at] = e + kept.size * 2.0 ** -24 + 2.0 ** -22 * abs(lse[at])
                    spread = (p / z) @ np.abs(v)
                    out_tol[at] = (2 * (e + 2.0 ** -weight_bits) + kept.size * 2.0 ** -23) * spread + kept.size * 2.0 ** -35 * np.abs(v).max(0) / z + 2.0 ** -out_bits * np.abs(out[at])
    return out, lse, out_tol, lse_tol


def attend_bf16(*args):
    return attend(*args, out_bits=8, weight_bits=11)


def attend_fp32(*args):
    return attend(*args, out_bits=23, weight_bits=22)


def as_double(t):
    if t.dtype == torch.float8_e4m3fn:
        t = t.float()
    return t.detach().double().cpu().numpy()
