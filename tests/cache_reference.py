"""The paged-cache operators and the token log probabilities from their
definitions in 64 bits, for the GPU tests; plain loops over requests and rows."""
import math

import torch

U = 2.0 ** -24  # unit roundoff of fp32


def place(table, x, P):
    """(page, row) of position x in a request's row of the block table."""
    return int(table[x // P]), x % P


def lines(cache, table_row, n, P):
    """The first n positions' lines [kv_heads, n, D] of a request, in 64 bits."""
    pages = table_row[: -(-n // P)].long()
    return cache[pages].double().transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])[:, :n]


def attend(q, key, value, table, ctx, new, mask, scale):
    """out, lse, and for the error bound: A = sum w |v| and S = the largest sum |q_i k_i| |scale| of a row
    (over all places of the request).  Keys and values of the requests' places are finite."""
    B, T, Hq, D = q.shape
    H, P = key.shape[1], key.shape[2]
    G = Hq // H
    out = torch.zeros((B, T, Hq, D), dtype=torch.float64, device=q.device)
    A = torch.zeros_like(out)
    lse = torch.full((B, T, Hq), -math.inf, dtype=torch.float64, device=q.device)
    S = torch.zeros_like(lse)
    for b in range(B):
        n, c = int(new[b]), int(ctx[b])
        if n == 0:
            continue
        k, v = lines(key, table[b], c + n, P), lines(value, table[b], c + n, P)
        seen = torch.ones((n, c + n), dtype=torch.bool, device=q.device)
        seen[:, c:] = torch.ones((n, n), device=q.device).tril() > 0 if mask is None else mask[b, :n, :n] != 0
        some = seen.any(1)
        for h in range(H):
            qs = q[b, :n, h * G:(h + 1) * G].double()                    # [n, G, D]
            x = (qs @ k[h].T * scale).masked_fill(~seen[:, None], -math.inf)
            w = torch.softmax(x, -1)
            w[~some] = 0
            out[b, :n, h * G:(h + 1) * G] = w @ v[h]
            A[b, :n, h * G:(h + 1) * G] = w @ v[h].abs()
            lse[b, :n, h * G:(h + 1) * G] = torch.logsumexp(x, -1)
            S[b, :n, h * G:(h + 1) * G] = (qs.abs() @ k[h].abs().T).amax(-1) * abs(scale)
    return out, lse, A, S


def attend_bounds(out, lse, A, S, D, L, bf16):
    """Elementwise bounds of the error.  A score is a sum of D fp32 products: off by at most (D + 8) U S, twice that
    relatively in a weight over its sum; sums over L keys add (L + 64) U; matrix units may truncate where the fp32
    units round, so all of it counts four times.  bf16: the weights and the result are rounded to 8 bits (unit roundoff 2^-8)."""
    d = (D + 8) * U * S
    rel = 4 * (2 * d + (L + 64) * U)
    e = rel[..., None] * A + 2.0 ** -60
    if bf16:
        e = e + 1.01 * 2.0 ** -8 * (A + out.abs())
    return e, 4 * (d + (L + 64) * U + U * lse.abs().nan_to_num(0, 0, 0)) + 1e-6


def rope(x, weight, eps, cos_sin, position, rot, interleaved):
    """x [heads, D] of one token: normed (weight not None) and rotated, in 64 bits."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    y = x.clone()
    for i in range(rot // 2):
        c, s = float(cos_sin[position, i]), float(cos_sin[position, rot // 2 + i])
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
    return y


def reserve(ctx, new, depth, table, owned, free, n_free, P, T, max_pages):
    """The free stack played through request by request; plain lists in and out."""
    table, owned, free = [list(r) for r in table], list(owned), list(free)
    B = len(ctx)
    fits = [c >= 0 and 0 <= n <= T and c + n <= max_pages * P for c, n in zip(ctx, new)]
    need = [-(-(c + n) // P) for c, n in zip(ctx, new)]
    top, dry, short = n_free, False, False
    for b in range(B):
        if fits[b] and owned[b] > need[b]:
            for j in range(need[b], owned[b]):
                free[top] = table[b][j]
                top += 1
            owned[b] = need[b]
    slot, position = [[-1] * T for _ in range(B)], [[-1] * T for _ in range(B)]
    left = top
    for b in range(B):
        want = need[b] - owned[b] if fits[b] else 0
        if want > 0:
            dry = dry or want > left
            if dry:
                short = True
                continue
            for j in range(owned[b], need[b]):
                left -= 1
                table[b][j] = free[left]
            owned[b] = need[b]
        if not fits[b]:
            continue
        for t in range(new[b]):
            page, row = place(table[b], ctx[b] + t, P)
            slot[b][t] = page * P + row
            position[b][t] = ctx[b] + (depth[b][t] if depth is not None else t)
    return table, owned, free, left, slot, position, short, not all(fits)


def logprobs(row, token, T, k):
    """log p(token), rank, entropy, top ids and their log probabilities of one row of logits."""
    x = row.double() + 0.0
    y = torch.log_softmax(x / T, 0)
    p = y.exp()
    order = torch.sort(x, descending=True, stable=True).indices
    top = [int(i) for i in order[:k] if x[i] > -math.inf]
    ids = top + [-1] * (k - len(top))
    lps = [float(y[i]) for i in top] + [-math.inf] * (k - len(top))
    rank = int((order == token).nonzero()[0, 0]) if token >= 0 else -1
    return float(y[token]) if token >= 0 else 0.0, rank, float(-(p * y)[p > 0].sum()), ids, lps
