"""The operators of a block with experts, plain numpy in 64 bits: written from their definitions (include/sparq_mx_experts.h) and shared by
the tests only."""
import numpy as np

import mx_reference as R


def sort(expert, experts):
    """offsets, place, order of the slots."""
    expert = np.asarray(expert).ravel()
    slots = [np.flatnonzero(expert == e) for e in range(experts)]
    offsets = np.cumsum([0] + [len(s) for s in slots])
    place, order = np.full(expert.size, -1), np.full(expert.size, -1)
    for e, s in enumerate(slots):
        place[s] = offsets[e] + np.arange(len(s))
        order[offsets[e]: offsets[e + 1]] = s
    return offsets, place, order


def gather(x, place, rows):
    """The rows that some slot has, and which these are."""
    y, has = np.zeros((rows, x.shape[1])), np.zeros(rows, bool)
    for t, row in enumerate(place):
        for p in row[(row >= 0) & (row < rows)]:
            y[p], has[p] = x[t], True
    return y, has


def combine(x, place, weights=None, residual=None):
    """y, and the sum of the terms' magnitudes."""
    tokens, per = place.shape
    y = np.zeros((tokens, x.shape[1]))
    size = np.zeros_like(y)
    for t in range(tokens):
        for j in range(per):
            if 0 <= place[t, j] < len(x):
                v = (1.0 if weights is None else weights[t, j]) * x[place[t, j]]
                y[t] += v
                size[t] += np.abs(v)
    return (y if residual is None else y + residual), (size if residual is None else size + np.abs(residual))


def combine_grad(dy, place, weights, x):
    """dx with which of its rows some slot has; dweights, and the sums of its terms' magnitudes."""
    dx, has = np.zeros((len(x), dy.shape[1])), np.zeros(len(x), bool)
    dw, size = np.zeros(place.shape), np.zeros(place.shape)
    for t in range(len(place)):
        for j, p in enumerate(place[t]):
            if 0 <= p < len(x):
                dx[p], has[p] = weights[t, j] * dy[t], True
                dw[t, j], size[t, j] = dy[t] @ x[p], np.abs(dy[t]) @ np.abs(x[p])
    return dx, has, dw, size


def ranges(offsets, rows):
    """Each expert's rows, cut off at the borders."""
    o = np.clip(np.asarray(offsets), 0, rows)
    return [(int(a), int(max(a, b))) for a, b in zip(o[:-1], o[1:])]


def product(A, W, offsets, bias=None):
    """z of the rows that an expert has, their sums' magnitudes, and which these are.  A [M][K] and W [experts][N][K]: values."""
    z, size, has = np.zeros((len(A), W.shape[1])), np.zeros((len(A), W.shape[1])), np.zeros(len(A), bool)
    for e, (a, b) in enumerate(ranges(offsets, len(A))):
        z[a:b] = A[a:b] @ W[e].T + (0 if bias is None else bias[e])
        size[a:b] = np.abs(A[a:b]) @ np.abs(W[e]).T + (0 if bias is None else np.abs(bias[e]))
        has[a:b] = True
    return z, size, has


def function(name, z):
    return z if name is None else R.function(name, z)


def random_words(groups, seed, offset):
    """Philox 4x32 with ten rounds: four words for each group, with whole numbers of any size."""
    out = []
    for g in groups:
        c = [g & 0xFFFFFFFF, g >> 32, offset & 0xFFFFFFFF, offset >> 32]
        k = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        out.append(c)
    return np.array(out, np.int64).reshape(-1, 4)


def kept(rows, K, p, seed, offset, first_row=0):
    """Which elements dropout keeps, and the rounded p."""
    limit = int(np.rint(p * 65536))
    per = -(-K // 8)
    w = random_words([(first_row + r) * per + i for r in range(rows) for i in range(per)], seed, offset % (1 << 64))
    bits = np.stack([w & 0xFFFF, w >> 16], -1).reshape(rows, per * 8)[:, :K]
    return bits >= limit, limit / 65536
