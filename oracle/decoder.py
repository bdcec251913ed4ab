"""Plain references, in 64 bits, of what stands around a decoder that makes its own logits and keeps a paged cache: selection from
dense logits, block tables, cache writes, attention.  TEST INFRASTRUCTURE: imported only by tests/; the product path never touches
it.  Python loops and numpy, from the definitions in include/lshbeam.h; no code is shared with the HIP path."""
from __future__ import annotations

import numpy as np

E4M3 = np.empty(256)
for _c in range(256):
    _e, _m = _c >> 3 & 15, _c & 7
    _v = (8 + _m) * 2.0 ** (_e - 10) if _e else _m * 2.0 ** -9
    E4M3[_c] = np.nan if _c & 127 == 127 else -_v if _c > 127 else _v
_MAGNITUDES = E4M3[:127]                     # 0 .. 448, ascending with their codes


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """Codes of the nearest e4m3 values, ties to even codes; NaN and infinities give NaN; |x| <= 448 otherwise."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(_MAGNITUDES, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _MAGNITUDES[hi] - a, a - _MAGNITUDES[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def select(logits, beam_scores, S, B, N, allowed=None):
    """(beam, word, score, lse, all scores [S, B, V]); logits [S*B, V], allowed truth values [S*B, V] or None."""
    x = np.asarray(logits, dtype=np.float64)
    if allowed is not None:
        x = np.where(allowed, x, -np.inf)
    with np.errstate(all="ignore"):
        top = x.max(axis=1, initial=-np.inf)
        shift = np.where(np.isfinite(top), top, 0.0)
        log_sum = np.log(np.exp(x - shift[:, None]).sum(axis=1))
        lse = shift + log_sum
        score = np.asarray(beam_scores, dtype=np.float64)[:, None] + ((x - shift[:, None]) - log_sum[:, None])
        score = np.where(np.isfinite(score.astype(np.float32)), score, -np.inf).reshape(S, B, -1)
    V = x.shape[1]
    beam, word, best = np.full((S, N), -1), np.full((S, N), -1), np.full((S, N), -np.inf)
    for s in range(S):
        flat = score[s].reshape(-1)
        order = np.argsort(-flat, kind="stable")[:N]
        order = order[np.isfinite(flat[order])]
        n = len(order)
        beam[s, :n], word[s, :n], best[s, :n] = order // V, order % V, flat[order]
    return beam, word, best, lse, score


def advance(S, B, T, n_blocks, block, tables, lengths, parents=None, n_new=None):
    """dict of tables, lengths, slots, copy_from, shared, status."""
    R, W = tables.shape
    rows = []
    for r in range(R):
        b = r % B if parents is None else int(parents[r])
        p = r - r % B + b if 0 <= b < B else -1
        old = int(lengths[p]) if p >= 0 else 0
        new = int(n_new[r]) if n_new is not None else (T if p >= 0 else 0)
        rows.append([p, old, new, [int(i) for i in tables[p, :-(-old // block)]] if p >= 0 else []])
    used = {i for _, _, _, t in rows for i in t}
    free = [i for i in range(n_blocks) if i not in used]
    refused = sum(new > T or old + new > W * block for _, old, new, _ in rows)
    copies, taken, want = [-1] * R, [], 0
    for r, (p, old, new, t) in enumerate(rows):
        if new and old % block:
            s0 = r - r % B
            if any(len(rows[q][3]) >= len(t) and rows[q][3][len(t) - 1] == t[-1] for q in range(s0, s0 + B) if q != r):
                copies[r] = t[-1]
        need = -(-(old + new) // block) - len(t) + (copies[r] >= 0)
        taken.append(need)
        want += need if not (new > T or old + new > W * block) else 0
    ok = refused == 0 and want <= len(free)
    out, slots, length = np.full((R, W), -1), np.full((R, T), -1), np.zeros(R, dtype=int)
    new_tables, at = [], 0
    for r, (p, old, new, t) in enumerate(rows):
        t, length[r] = list(t), old
        if ok:
            if copies[r] >= 0:
                t.pop()
            t += free[at:at + taken[r]]
            at += taken[r]
            length[r] = old + new
            for i in range(new):
                slots[r, i] = t[(old + i) // block] * block + (old + i) % block
        out[r, :len(t)] = t
        new_tables.append(t)
    shared = np.zeros(S, dtype=int)
    for s in range(S):
        mine = [r for r in range(s * B, s * B + B) if length[r] > 0]
        if mine:
            n = 0
            while all(n < length[r] // block for r in mine) and len({new_tables[r][n] for r in mine}) == 1:
                n += 1
            shared[s] = n
    return {"tables": out, "lengths": length, "slots": slots, "copy_from": np.array(copies if ok else [-1] * R), "shared": shared,
            "status": np.array([max(0, want - len(free)), refused])}


class Pool:
    """Codes in reading order: k, v [n_blocks, heads, block, D] uint8; scales [n_blocks, heads]."""

    def __init__(self, k, v, k_scale, v_scale):
        self.k, self.v = np.array(k), np.array(v)
        self.k_scale, self.v_scale = np.array(k_scale, dtype=np.float64), np.array(v_scale, dtype=np.float64)

    @classmethod
    def from_layout(cls, k, v, k_scale, v_scale):
        """From the arrays of a lsh_cache_pool."""
        n, h, c, bs, _ = k.shape
        return cls(k.transpose(0, 1, 3, 2, 4).reshape(n, h, bs, 16 * c), v.transpose(0, 1, 2, 4, 3).reshape(n, h, bs, 16 * c), k_scale, v_scale)

    def layout(self):
        n, h, bs, d = self.k.shape
        return (np.ascontiguousarray(self.k.reshape(n, h, bs, d // 16, 16).transpose(0, 1, 3, 2, 4)),
                np.ascontiguousarray(self.v.reshape(n, h, bs // 16, 16, d).transpose(0, 1, 2, 4, 3)))

    def values(self, which, block, h):
        return E4M3[getattr(self, which)[block, h]] * getattr(self, which + "_scale")[block, h]


def scale_for(amax):
    if amax == 0:
        return 0.0
    s = 2.0 ** -126
    while amax > 448 * s:
        s *= 2
    return s


def write(pool: Pool, k, v, slots, copy_from=None):
    """k, v [R, T, heads, D]; changes `pool`."""
    n_blocks, heads, bs, D = pool.k.shape
    before = Pool(pool.k, pool.v, pool.k_scale, pool.v_scale)
    for r in range(slots.shape[0]):
        t = 0
        while t < slots.shape[1] and slots[r, t] >= 0:
            b, at = divmod(int(slots[r, t]), bs)
            n = min(int((slots[r, t:] >= 0).sum()), bs - at)
            src = int(copy_from[r]) if t == 0 and at > 0 and copy_from is not None and copy_from[r] >= 0 else b
            for name, x in (("k", k), ("v", v)):
                codes, scales, old, old_scales = getattr(pool, name), getattr(pool, name + "_scale"), getattr(before, name), getattr(before, name + "_scale")
                for h in range(heads):
                    new = np.asarray(x[r, t:t + n, h], dtype=np.float64)
                    fin = np.abs(new[np.isfinite(new)])
                    was = old_scales[src, h] if at else 0.0
                    s = max(was, scale_for(fin.max() if fin.size else 0.0))
                    if at:                   # a scale that stays leaves the codes as they are (those of a block of zeros too)
                        codes[b, h, :at] = old[src, h, :at] if was == s else to_e4m3(E4M3[old[src, h, :at]] * (was / s))
                    with np.errstate(all="ignore"):
                        codes[b, h, at:at + n] = to_e4m3(new / s if s else np.where(np.isfinite(new), 0.0 * new, np.nan))
                    scales[b, h] = s
            t += n


def attention(pool: Pool, q, tables, lengths, scale, causal=True, window=0, n_new=None):
    """(out, lse, how large: sum p |v|, sum |q k| scale of the largest product); q [R, T, heads, D]; tokens behind n_new are NaN."""
    R, T, Hq, D = q.shape
    heads, bs = pool.k.shape[1], pool.k.shape[2]
    out, lse = np.full((R, T, Hq, D), np.nan), np.full((R, T, Hq), np.nan)
    size, reach = np.zeros((R, T, Hq, D)), np.zeros((R, T, Hq))
    for r in range(R):
        L = int(lengths[r])
        n = T if n_new is None else int(n_new[r])
        for h in range(Hq):
            g = h // (Hq // heads)
            ids = [int(i) for i in tables[r, :-(-L // bs)]]
            k = np.concatenate([pool.values("k", i, g) for i in ids] + [np.zeros((0, D))])[:L]
            v = np.concatenate([pool.values("v", i, g) for i in ids] + [np.zeros((0, D))])[:L]
            for t in range(n):
                hi = max(0, L - n + t + 1) if causal else L
                lo = max(0, hi - window) if window else 0
                if lo >= hi:
                    out[r, t, h], lse[r, t, h] = 0.0, -np.inf
                    continue
                x = np.asarray(q[r, t, h], dtype=np.float64)
                s = k[lo:hi] @ x * scale
                m = s.max()
                p = np.exp(s - m)
                lse[r, t, h] = m + np.log(p.sum())
                out[r, t, h] = p @ v[lo:hi] / p.sum()
                size[r, t, h] = p @ np.abs(v[lo:hi]) / p.sum()
                reach[r, t, h] = (np.abs(k[lo:hi]) @ np.abs(x)).max() * scale
    return out, lse, size, reach
