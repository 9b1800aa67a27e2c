"""The 4-bit cache, the rotation and attention over the cache, written plainly in numpy: what the tests compare with."""
import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
PAGE = 16


def run_bytes(D):
    return 17 * D // 2


def quantise(x):
    """Codes [..., D] and scale bytes [..., D/32] of float32 rows, in 64 bits."""
    x = np.asarray(x, np.float32)
    y = x.reshape(*x.shape[:-1], -1, 32).astype(np.float64)
    top = np.abs(y).max(-1)
    none = ~np.isfinite(y).all(-1)
    safe = np.where(none | (top == 0), 1.0, top)
    m, e = np.frexp(safe)                                  # m in [0.5, 1): the largest is 2 m 2^(e - 1)
    byte = np.clip(e - 1 - 2 + (2 * m > 1.75) + 127, 2, 252)
    byte = np.where(top == 0, 2, byte)
    size = np.abs(np.where(none[..., None], 0, y)) * np.exp2(127.0 - byte)[..., None]
    near = np.abs(size[..., None] - GRID)
    code = near.argmin(-1)                                 # a tie goes to the smaller code; the even one is wanted
    tie = (code < 7) & (np.take_along_axis(near, code[..., None], -1)[..., 0] == np.take_along_axis(near, np.minimum(code + 1, 7)[..., None], -1)[..., 0])
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = np.where(none[..., None], 0, code | np.where(np.signbit(y), 8, 0))
    byte = np.where(none, 255, byte)
    return code.reshape(x.shape).astype(np.uint8), byte.astype(np.uint8)


def dequantise(code, byte):
    v = np.where(code & 8, -GRID[code & 7], GRID[code & 7]).reshape(*code.shape[:-1], -1, 32)
    scale = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return (v * scale[..., None]).reshape(code.shape)


def element_at(D, values):
    """Number of element (token, d) within a run's elements, [16, D]."""
    t, d = np.arange(16)[:, None], np.arange(D)[None]
    part = D // 16
    return ((t // 4 * 16 + d // part) * 4 + t % 4) * part + d % part if values else t * D + d


def write_row(run, D, values, token, code, byte):
    """One token's codes [D] and scale bytes [D/32] into a run's bytes (a view)."""
    at = element_at(D, values)[token]
    for d in range(D):
        i, shift = at[d] // 2, 4 * (at[d] % 2)
        run[i] = (run[i] & (0xF0 >> shift)) | (int(code[d]) << shift)
    run[8 * D + np.arange(D // 32) * 16 + token] = byte


def read_runs(run, D, values):
    """Runs [..., 17 D / 2] -> codes [..., 16, D] and scale bytes [..., 16, D/32]."""
    at = element_at(D, values)
    code = (run[..., at // 2] >> (4 * (at % 2)).astype(np.uint8)) & 15
    return code, np.moveaxis(run[..., 8 * D:].reshape(*run.shape[:-1], D // 32, 16), -1, -2)


def pack_runs(code, byte, values):
    """Codes [..., 16, D] and scale bytes [..., 16, D/32] -> runs."""
    D = code.shape[-1]
    flat = np.zeros((*code.shape[:-2], 16 * D), np.uint8)
    flat[..., element_at(D, values).ravel()] = code.reshape(*code.shape[:-2], -1)
    return np.concatenate([flat[..., 0::2] | (flat[..., 1::2] << 4), np.moveaxis(byte, -2, -1).reshape(*byte.shape[:-2], -1)], -1)


def rotate32(x, cos_sin, pos, interleaved):
    """Rows [T,H,D] of float32, every product and sum rounded to float32."""
    x = np.asarray(x, np.float32)
    R = cos_sin.shape[1]
    cos, sin = cos_sin[pos, None, :R // 2], cos_sin[pos, None, R // 2:]
    lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    out = x.copy()
    out[..., lo], out[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., hi] * cos + x[..., lo] * sin
    return out


def rotate64(x, cos_sin, pos, interleaved):
    """The same in 64 bits, and the sum of the two products' magnitudes (what their roundings are relative to)."""
    x, cs = np.asarray(x, np.float64), cos_sin.astype(np.float64)
    R = cs.shape[1]
    cos, sin = cs[pos, None, :R // 2], cs[pos, None, R // 2:]
    lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    out, size = x.copy(), np.zeros_like(x)
    out[..., lo], out[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., hi] * cos + x[..., lo] * sin
    size[..., lo], size[..., hi] = abs(x[..., lo] * cos) + abs(x[..., hi] * sin), abs(x[..., hi] * cos) + abs(x[..., lo] * sin)
    return out, size


def random_tree(rng, n, max_depth=12):
    parent, depth = np.full(n, -1), np.zeros(n, int)
    for i in range(1, n):
        up = i - 1 if rng.random() < 0.5 and depth[i - 1] < max_depth else int(rng.integers(0, i))
        parent[i], depth[i] = up, depth[up] + 1
    return parent, depth


def tree_mask(parent, K):
    """[K,2] uint64 words of the ancestor bits."""
    bits = np.zeros((K, 2), np.uint64)
    for i, p in enumerate(parent):
        if p >= 0:
            bits[i] = bits[p]
        bits[i, i // 64] |= np.uint64(1) << np.uint64(i % 64)
    return bits


def attention(q, k, v, see, scale, cap):
    """q [n,G,D], k, v [L,D] in 64 bits, see [n,L]: rows, and how far a kernel's may be from them.

    The bound, element by element: probabilities are rounded to bfloat16 (half a step is 2^-8 of each at most), scores are off by
    delta = |scale| sum over blocks of 2^-14 max|q| sum|k| (what three 6-bit numbers leave out of a query), plus 2^-17 of the sum of the
    products' magnitudes (128 fp32 sums of half a step 2^-24 each) and 2^-16 for the argument of exp2, exp2 itself and, with a cap,
    its tanh (relative to the cap: a few steps of 2^-23); a relative error e of all weights moves the mean by at most
    2 e sum p|v| / sum p, of which rounding's half shows in numerator alone; the result is rounded to bfloat16."""
    n, G, D = q.shape
    with np.errstate(invalid="ignore"):
        x = np.einsum("ngd,ld->ngl", q, k) * scale
        off = abs(scale) * (2.0 ** -14 * np.einsum("ngb,lb->ngl", abs(q).reshape(n, G, -1, 32).max(-1), np.nan_to_num(abs(k)).reshape(len(k), -1, 32).sum(-1))
                            + 2.0 ** -17 * np.einsum("ngd,ld->ngl", abs(q), np.nan_to_num(abs(k))))
        if cap:
            x = cap * np.tanh(x / cap)
            off = off + cap * 2.0 ** -20
        x = np.where(see[:, None], x, -np.inf)
        off = np.where(see[:, None], off, 0)
        top = x.max(-1, keepdims=True, initial=-np.inf)
        p = np.where(np.isfinite(top), np.exp(x - np.where(np.isfinite(top), top, 0)), 0)
        p = np.where(np.isnan(x), np.nan, p)
    total = p.sum(-1, keepdims=True)
    weight = p / np.where(total == 0, 1, total)
    seen_v = np.where(see[:, None, :, None], v[None, None], 0) if np.isnan(v).any() else None
    out = np.einsum("ngl,ngld->ngd", weight, np.broadcast_to(seen_v, (n, G, *v.shape))) if seen_v is not None else np.einsum("ngl,ld->ngd", weight, v)
    mean = np.einsum("ngl,ld->ngd", np.nan_to_num(weight), np.nan_to_num(abs(v)))
    e = off.max(-1, keepdims=True, initial=0) + 2.0 ** -16
    tol = (2.0 ** -8 + 2 * np.expm1(e)) * mean + 2.0 ** -8 * np.nan_to_num(abs(out)) + 1e-37
    return out, tol
