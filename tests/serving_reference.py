"""Plain references of the serving operators in 64 bits (numpy, on the host), and the batches that their tests use."""
import numpy as np

BF16_STEP = 2.0 ** -8    # a rounding to bf16 is off by at most this, relative to the value
FP32_STEP = 2.0 ** -24


def f64(t):
    return t.detach().double().cpu().numpy()


def attention(q, k_cache, v_cache, pages, row_start, kv_len, page, scale, causal=True):
    """q [rows, H, hd], caches [pages, Hkv, page, hd].  Returns (out, sum of p |v|, largest sum of |q k|), out NaN-free for
    rows of no sequence (zero)."""
    rows, H, hd = q.shape
    Hkv = k_cache.shape[1]
    G = H // Hkv
    out, weight, score = np.zeros((rows, H, hd)), np.zeros((rows, H, hd)), 0.0
    for b in range(len(kv_len)):
        n, kv = int(row_start[b + 1] - row_start[b]), int(kv_len[b])
        where = np.arange(kv)
        pg = pages[b][where // page] if kv else where
        for h in range(Hkv):
            K, V = k_cache[pg, h, where % page], v_cache[pg, h, where % page]
            for i in range(n):
                pos = kv - n + i
                seen = 0 if pos < 0 else (pos + 1 if causal else kv)
                if seen == 0:
                    continue
                for c in range(h * G, (h + 1) * G):
                    r = row_start[b] + i
                    s = scale * (K[:seen] @ q[r, c])
                    score = max(score, abs(scale) * np.max(np.abs(K[:seen]) @ np.abs(q[r, c])))
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    out[r, c] = p @ V[:seen]
                    weight[r, c] = p @ np.abs(V[:seen])
    return out, weight, score


def attention_bound(ref, weight, score, hd, keys, bf16):
    """How far a right result may be off, element by element.  Scores: a sum of hd products in fp32 and two more roundings,
    so their error is at most (hd + 2) * 2^-24 * sum|q k|; the reference of the exponents and its product add two steps
    of the largest score each, the exponential four; an error d of a score changes a weight by the factor exp(2 d) at most
    (its own and the normalisation's).  The weighted sum adds `keys` steps.  bf16: one rounding per probability, and one of
    the result.  Where the sum that normalises is that of the rounded probabilities p (1 + e), |e| <= 2^-8, the result is off
    by sum p e (v - out) / sum p (1 + e): at most 2^-8 (sum p |v| + |out|) and a factor 1 / (1 - 2^-8)."""
    d = (hd + 2) * FP32_STEP * score + 4 * FP32_STEP * score + 4 * FP32_STEP
    tol = weight * (np.expm1(2 * d) + (2 * keys + 8) * FP32_STEP)
    if bf16:
        tol = tol + (weight + np.abs(ref)) * BF16_STEP / (1 - BF16_STEP)
    return tol + (np.abs(ref) + tol) * (BF16_STEP if bf16 else FP32_STEP) + 1e-37


def frequencies(rotary_dim, theta, scaling, factor=1.0, low=1.0, high=32.0, original_len=1):
    f = theta ** (-2.0 * np.arange(rotary_dim // 2) / rotary_dim)
    if scaling == "linear":
        return f / factor
    if scaling == "by_parts":
        w = np.clip((original_len * f / (2 * np.pi) - low) / (high - low), 0, 1)
        return f * (w + (1 - w) / factor)
    return f


def rotate(x, pos, freq, layout, magnitude=1.0):
    """x [rows, heads, hd], pos [rows]."""
    y = x.copy()
    h = len(freq)
    a, b = (np.arange(h), np.arange(h) + h) if layout == "half" else (2 * np.arange(h), 2 * np.arange(h) + 1)
    z = (x[..., a] + 1j * x[..., b]) * (magnitude * np.exp(1j * np.asarray(pos, float)[:, None] * freq))[:, None]
    y[..., a], y[..., b] = z.real, z.imag
    return y


def positions(row_start, kv_len):
    pos = []
    for b in range(len(kv_len)):
        n = int(row_start[b + 1] - row_start[b])
        pos += [int(kv_len[b]) - n + i for i in range(n)]
    return np.array(pos, dtype=np.int64)


def sample(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """One row: the definition, step by step."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, dtype=np.float64))
    top = x.max()
    if top == -np.inf:
        return -1
    if not T > 0:
        return int(np.argmax(x))
    w = np.where(x == top, 1.0, np.exp(np.where(x == top, 0.0, x - top) / T)) if np.isfinite(top) else (x == top).astype(float)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if 0 < k < len(x):
        order = order[:k]
    if p < 1:
        c = np.cumsum(w[order])
        order = order[:1 + np.count_nonzero(c[:-1] < p * c[-1])]
    if m > 0:
        order = order[w[order] >= m]
    order = np.sort(order)
    c = np.cumsum(w[order])
    return int(order[min(np.searchsorted(c, u * c[-1], side="right"), np.flatnonzero(w[order])[-1])])


def page_table(rng, kv_len, page, spare=3, width=None):
    """Shuffled pages: (table [n, width], pages in the pool).  Entries behind a sequence's last page are nonsense."""
    need = [(int(k) + page - 1) // page for k in kv_len]
    total = sum(need) + spare
    order = rng.permutation(total)
    table = np.full((len(need), width or max(max(need), 1)), -77, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total
