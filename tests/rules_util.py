"""The rules of graft_logits_adjust and graft_token_counts in plain numpy, each fp32 operation rounded by itself."""
import numpy as np

PROMPT = np.int32(-2 ** 31)


def counts_of(ctx, ctx_len, prompt_len, V, start=None, counts=None):
    """graft_token_counts: (counts, status)."""
    B, L = ctx.shape
    out = np.zeros((B, V), np.int32) if counts is None or start is None else counts.copy()
    status = np.zeros(B, np.int32)
    for b in range(B):
        s, n = 0 if start is None else int(start[b]), int(ctx_len[b])
        if not (0 <= n <= L and 0 <= s <= n):
            status[b] = 1
            continue
        for t in range(s, n):
            v = int(ctx[b, t])
            if not 0 <= v < V:
                continue
            if prompt_len is not None and t < prompt_len[b]:
                out[b, v] |= PROMPT
            else:
                out[b, v] += np.int32(1)
    return out, status


def adjusted(logits, n_nodes, tokens=None, mask=None, counts=None, repetition=None, frequency=None, presence=None, bias=None, allow=None,
             allow_index=None):
    """(logits under the rules, padding rows as they were; target ids; status)."""
    B, K, V = logits.shape
    out, ids, status = logits.copy(), np.full((B, K), -1, np.int32), np.zeros(B, np.int32)
    f32 = np.float32
    with np.errstate(all="ignore"):
        for b in range(B):
            n = int(n_nodes[b])
            if not 1 <= n <= K:
                status[b] = 2
                continue
            for i in range(n):
                x = logits[b, i].copy()
                c = np.zeros(V, np.int64) if counts is None else counts[b].astype(np.int64)
                later, seen = c & 0x7FFFFFFF, c < 0
                if mask is not None:
                    for j in range(1, n):
                        if (int(mask[b, i, j // 64]) >> (j % 64)) & 1 and 0 <= tokens[b, j] < V:
                            later[tokens[b, j]] += 1
                gen = later > 0
                if repetition is not None:
                    x = np.where(seen | gen, np.where(x > 0, x / f32(repetition[b]), x * f32(repetition[b])), x)
                if frequency is not None:
                    x = np.where(gen, x - later.astype(f32) * f32(frequency[b]), x)
                if presence is not None:
                    x = np.where(gen, x - f32(presence[b]), x)
                if bias is not None:
                    x = x + (bias if bias.ndim == 1 else bias[b])
                if allow is not None:
                    at = int(allow_index[b, i])
                    if not -1 <= at < len(allow):
                        status[b] |= 1
                        x = np.full(V, -np.inf, f32)
                    elif at >= 0:
                        v = np.arange(V)
                        x = np.where((allow[at].view(np.uint32)[v // 32] >> (v % 32).astype(np.uint32)) & 1, x, f32(-np.inf))
                out[b, i] = x
                y = np.where(np.isnan(x), -np.inf, x)
                ids[b, i] = int(y.argmax()) if y.max() > -np.inf else -1
    return out, ids, status
