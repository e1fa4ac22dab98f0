"""The rollout step's operators from their definitions (test infrastructure): quantised rows, attention over a
sequence's keys and values in 64 bits, verification of drafted tokens.  Plain loops over sequences and heads."""
import numpy as np

from . import quant
from .cast import BF16, F32, f32_to_bf16_bits, bf16_to_f32_bits


def quantize_row(x: np.ndarray):
    """(codes, scale) of one fp32 row: the bucket rule of `quant` with the row as the tensor."""
    bits = np.asarray(x, np.float32).view(np.uint32)
    amax = quant.amax_bits(bits, F32)
    s, r = quant.scale_of(amax), quant.rscale_of(amax)
    return quant.quantize(bits, F32, s, r), s


def dequantize_row(codes: np.ndarray, scale: np.float32) -> np.ndarray:
    return quant.dequantize(codes, F32, scale).view(np.float32)


def to_bf16(x: np.ndarray) -> np.ndarray:
    """fp32 values rounded to bf16, as fp32."""
    return bf16_to_f32_bits(f32_to_bf16_bits(np.asarray(x, np.float32).view(np.uint32))).view(np.float32)


def attend(q, keys, values, n_new, scale, window=0):
    """Attention of a sequence's last `n_new` tokens over its keys and values, fp64.

    q [n_new, heads, D]; keys, values [kv_heads, length, D]; the position of new token i is length - n_new + i and
    may be negative (a row with nothing to attend over).  Returns (out, lse, weight): weight[i, h, d] =
    sum_j softmax_j |value_j,d|, the scale of the rounding that a 16-bit softmax weight brings."""
    n, heads, d = q.shape
    kv_heads, length, _ = keys.shape
    g = heads // kv_heads
    out = np.zeros((n, heads, d))
    mag = np.zeros((n, heads, d))
    lse = np.full((n, heads), -np.inf)
    for i in range(n):
        pos = length - n_new + i
        lo = max(0, pos - window + 1) if window else 0
        if pos < lo or pos < 0:
            continue
        for h in range(heads):
            k = keys[h // g, lo:pos + 1].astype(np.float64)
            v = values[h // g, lo:pos + 1].astype(np.float64)
            z = (k @ q[i, h].astype(np.float64)) * scale
            top = z.max()
            if top == -np.inf:
                continue
            w = np.exp(z - top)
            total = w.sum()
            lse[i, h] = top + np.log(total)
            out[i, h] = (w / total) @ v
            mag[i, h] = (w / total) @ np.abs(v)
    return out, lse, mag


def verify(target, draft, tokens, uniform, race, max_drafts):
    """One sequence: (accepted, emitted tokens padded with -1 to max_drafts + 1).  All fp32 arithmetic, one rounding
    per operation."""
    k, vocab = len(tokens), target.shape[1]
    a = 0
    with np.errstate(invalid="ignore", divide="ignore", over="ignore", under="ignore"):
        while a < k:
            x = int(tokens[a])
            if not 0 <= x < vocab:
                break
            q = np.float32(1.0) if draft is None else np.float32(draft[a, x])
            if not np.float32(uniform[a]) * q < np.float32(target[a, x]):
                break
            a += 1
        p = target[a].astype(np.float32)
        w = p.copy()
        if a < k:
            if draft is not None:
                w = p - draft[a].astype(np.float32)
            elif 0 <= int(tokens[a]) < vocab:
                w[int(tokens[a])] = 0
        for weights in (w, p):
            best, token = np.float32(-1.0), 0
            for v in np.flatnonzero(weights > 0):
                score = np.float32(weights[v]) / np.float32(race[v])
                if score > best:
                    best, token = score, int(v)
            if best >= 0:
                break
    out = np.full(max_drafts + 1, -1, np.int32)
    out[:a] = tokens[:a]
    out[a] = token
    return a, out


# ---- trees of drafted tokens ---------------------------------------------------------------------
def ancestors(parent):
    """Per row of a tree, the rows it continues (nearest first) behind itself."""
    out = []
    for i, p in enumerate(parent):
        out.append([i] + (out[p] if 0 <= p < i else []))
    return out


def turn(x, cos, sin, interleaved=False):
    """A row's first 2 len(cos) elements turned in pairs, each product and sum rounded to fp32 by itself."""
    x = np.asarray(x, np.float32)
    y, half = x.copy(), len(cos)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def attend_rows(q, keys, values, sees, scale):
    """attend() with the positions that each row sees as a table [n_new, length] of truth values."""
    n, heads, d = q.shape
    g = heads // keys.shape[0]
    out, mag, lse = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.full((n, heads), -np.inf)
    for i in range(n):
        at = np.flatnonzero(sees[i])
        if not len(at):
            continue
        for h in range(heads):
            k, v = keys[h // g, at].astype(np.float64), values[h // g, at].astype(np.float64)
            z = (k @ q[i, h].astype(np.float64)) * scale
            top = z.max()
            if top == -np.inf:
                continue
            w = np.exp(z - top)
            total = w.sum()
            lse[i, h] = top + np.log(total)
            out[i, h] = (w / total) @ v
            mag[i, h] = (w / total) @ np.abs(v)
    return out, lse, mag


def tree_sees(bits, length, window=0):
    """The positions that rows of a tree see, from `bits` [n_new, n_new] (which of the new rows up to its own)."""
    n = len(bits)
    first = length - n
    sees = np.zeros((n, length), bool)
    for i in range(n):
        mine = np.flatnonzero(bits[i][:i + 1])
        low = max(0, first + len(mine) - window) if window else 0
        sees[i, low:max(first, 0)] = True
        for j in mine:
            if first + j >= 0:
                sees[i, first + j] = True
    return sees


def verify_tree(target, draft, tokens, parent, uniform, race, max_depth):
    """One tree: (accepted rows, emitted tokens).  fp32 arithmetic, one rounding per operation; sums in 64 bits."""
    n, vocab = len(parent), target.shape[1]
    f32 = np.float32
    if n == 0:
        return [], []
    here, path, emitted = 0, [], []
    with np.errstate(invalid="ignore", divide="ignore", over="ignore", under="ignore"):
        while True:
            p = target[here].astype(f32)
            left, mass, moved, kids = p.copy(), f32(1), False, 0
            if len(path) < max_depth:
                for c in range(here + 1, n):
                    x = int(tokens[c])
                    if parent[c] != here or not 0 <= x < vocab:
                        continue
                    if kids == 256:
                        break
                    kids += 1
                    q = f32(1) if draft is None else f32(draft[here, x])
                    if f32(uniform[c]) * (mass * q) < left[x]:
                        here, moved = c, True
                        path.append(c)
                        emitted.append(x)
                        break
                    if draft is None:
                        mass = np.fmax(mass - left[x], f32(0))
                        left[x] = 0
                    else:
                        left = np.fmax(left - mass * draft[here].astype(f32), f32(0))
                        mass = f32(left.astype(np.float64).sum())
            if moved:
                continue
            for weights in (left, p):
                best, token = f32(-1), 0
                for v in np.flatnonzero(weights > 0):
                    score = f32(weights[v]) / f32(race[v])
                    if score > best:
                        best, token = score, int(v)
                if best >= 0:
                    break
            return path, emitted + [token]
