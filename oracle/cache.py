"""Context-cache oracle: windowed attention, 4-bit values, slot weights, eviction.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``).

Plain numpy float64, one element or one row at a time where that is the
definition:

* ``visible``    which keys a new row sees: with a window W > 0 the context slots
  j with j < n_sinks or position - j < W, of a tree's new keys the ancestors
  for which the same holds at their positions (ctx + depth), of a block's all;
* ``encode`` / ``decode``  4-bit values: 32 dims share 2^e, each the nearest of
  0, .5, 1, 1.5, 2, 3, 4, 6 times 2^e by distance (ties to the even code);
* ``attention``  softmax attention over [context ; new keys] with that mask;
* ``weigh``      the attention weight each slot receives, added to old weights;
* ``evict``      the slots that a budget keeps.
"""

import math

import numpy as np

from .attention import _f64, _i64, tree_visibility

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK = 32
MIN_EXP, MAX_EXP = -125, 125


def depths(parents):
    return tree_visibility(parents).sum(1) - 1


def visible(ctx, n, parents=None, n_sinks=0, window=0):
    """Bool [n][ctx + n]: new row i sees key j (context slots, then new rows)."""
    anc = np.ones((n, n), dtype=bool) if parents is None else tree_visibility(parents)
    depth = np.arange(n) if parents is None else depths(parents)
    vis = np.ones((n, ctx + n), dtype=bool)
    vis[:, ctx:] = anc
    if window:
        for i in range(n):
            pos = ctx + depth[i]
            for j in range(ctx):
                vis[i, j] = j < n_sinks or pos - j < window
            if parents is not None:
                for k in range(n):
                    at = ctx + depth[k]
                    vis[i, ctx + k] &= at < n_sinks or pos - at < window
    return vis


def block_exponent(values):
    """e of a block: floor(log2 a) - 2, one more if a >= 1.75 2^floor(log2 a), within MIN_EXP..MAX_EXP;
    None if the block holds a NaN or an infinity."""
    a = np.abs(values).max()
    if not np.isfinite(values).all():
        return None
    if a == 0:
        return MIN_EXP
    m, x = math.frexp(a)  # a = m 2^x, m in [0.5, 1)
    return min(MAX_EXP, max(MIN_EXP, x - 1 - 2 + (1 if 2 * m >= 1.75 else 0)))


def encode(x):
    """Codes (uint8, one per value) and scale bytes of [..., d] values."""
    x = _f64(x)
    blocks = x.reshape(-1, BLOCK)
    codes = np.zeros(blocks.shape, dtype=np.uint8)
    scales = np.zeros(len(blocks), dtype=np.uint8)
    grid = np.array(GRID)
    even_first = np.argsort([c % 2 for c in range(8)], kind="stable")  # even codes win equal distances
    exps = [block_exponent(v) for v in blocks]
    scales[:] = [255 if e is None else e + 127 for e in exps]
    fine = scales != 255
    v = blocks[fine] * 2.0 ** -(scales[fine].astype(np.float64) - 127)[:, None]
    dist = np.abs(np.abs(v)[..., None] - grid[even_first])
    codes[fine] = even_first[dist.argmin(-1)] + 8 * np.signbit(v)
    return codes.reshape(x.shape), scales.reshape(*x.shape[:-1], -1)


def pack(codes):
    """Two codes a byte, the even dim in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def decode(packed, scales):
    """float64 values of packed codes and scale bytes."""
    packed, scales = np.asarray(packed), np.asarray(scales)
    codes = np.empty((*packed.shape[:-1], 2 * packed.shape[-1]), dtype=np.int64)
    codes[..., 0::2], codes[..., 1::2] = packed & 15, packed >> 4
    v = np.array(GRID + tuple(-g for g in GRID))[codes]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


def _scores(q, k, k_new, sm_scale):
    """Scaled scores [hq][n][keys] of one sequence."""
    n, hq, d = q.shape
    group = hq // k.shape[0]
    scale = sm_scale if sm_scale and sm_scale > 0 else 1.0 / math.sqrt(d)
    keys = [np.concatenate([k[g], k_new[:, g]]) for g in range(k.shape[0])]
    return np.stack([scale * (q[:, h] @ keys[h // group].T) for h in range(hq)])


def attention(q, k, v, k_new, v_new, lens, parents=None, n_sinks=0, window=0, sm_scale=None):
    """Batched.  k, v [batch][Hkv][cap][D]; q, k_new, v_new [batch][n][H][D].  Context slots that no
    row sees are never touched (they may hold anything)."""
    q, k, v, k_new, v_new = (_f64(t) for t in (q, k, v, k_new, v_new))
    batch, n, hq, d = q.shape
    group = hq // k.shape[1]
    out, lse = np.zeros(q.shape), np.zeros((batch, n, hq))
    for b, ctx in enumerate(_i64(lens)):
        vis = visible(ctx, n, None if parents is None else parents[b], n_sinks, window)
        use = vis.any(0)
        use[ctx:] = True
        at = np.flatnonzero(use[:ctx])
        kb, vb, m = k[b][:, at], v[b][:, at], vis[:, use]
        s = np.where(m[None], _scores(q[b], kb, k_new[b], sm_scale), -np.inf)
        top = s.max(-1, keepdims=True)
        e = np.exp(s - top)
        total = e.sum(-1, keepdims=True)
        lse[b] = (top + np.log(total))[..., 0].T
        for h in range(hq):
            vals = np.concatenate([vb[h // group], v_new[b][:, h // group]])
            out[b, :, h] = e[h] @ vals / total[h]
    return out, lse


def path_nodes(accept_len, accept_path, n):
    """The nodes a commit takes: up to accept_len + 1, stopping at the first that is none."""
    nodes = []
    for t in range(min(int(accept_len) + 1, len(accept_path), n)):
        if not 0 <= int(accept_path[t]) < n:
            break
        nodes.append(int(accept_path[t]))
    return nodes


def weigh(q, k, lse, lens, weights, decay=1.0, k_new=None, accept_len=None, accept_path=None, n_sinks=0, window=0,
          sm_scale=None):
    """New weights [batch][Hkv][cap].  Without a path the rows are a block's."""
    q, k, lse = (_f64(t) for t in (q, k, lse))
    out = np.array(_f64(weights), copy=True)
    batch, n, hq, _ = q.shape
    hkv, cap = k.shape[1], k.shape[2]
    group = hq // hkv
    for b, ctx in enumerate(_i64(lens)):
        nodes = list(range(n)) if accept_path is None else path_nodes(accept_len[b], accept_path[b], n)
        rows = len(nodes)
        new = np.zeros((rows, hkv, q.shape[3])) if k_new is None else _f64(k_new[b])[nodes]
        # the path's rows are a chain: positions ctx + t, each row sees itself and those before it
        vis = visible(ctx, rows, None if accept_path is None else list(range(-1, rows - 1)), n_sinks, window) \
            if rows else np.zeros((0, ctx), dtype=bool)
        if rows:
            s = np.where(vis[None], _scores(q[b][nodes], k[b][:, :ctx], new, sm_scale), -np.inf)
            p = np.exp(s - lse[b][nodes].T[..., None])
            p = p.reshape(hkv, group, rows, -1).sum((1, 2))
        else:
            p = np.zeros((hkv, ctx))
        old = decay * out[b, :, :ctx] if decay else 0.0
        out[b, :, :ctx] = old + p[:, :ctx]
        if accept_path is not None:
            for t in range(rows):
                if ctx + t < cap:
                    out[b, :, ctx + t] = p[:, ctx + t]
    return out


def evict(lens, weights, budget, n_sinks=0, n_recent=0):
    """kept[b][g]: the slots kept of every sequence and KV head, ascending."""
    kept = []
    for b, ctx in enumerate(_i64(lens)):
        per_head = []
        for w in np.asarray(weights)[b]:
            if ctx <= budget:
                per_head.append(list(range(ctx)))
                continue
            middle = range(n_sinks, ctx - n_recent)
            key = [math.inf if math.isnan(x) else float(x) for x in w]
            order = sorted(middle, key=lambda j: (not math.isnan(w[j]), -key[j], j))
            take = order[:budget - n_sinks - n_recent]
            per_head.append(sorted([*range(n_sinks), *take, *range(ctx - n_recent, ctx)]))
        kept.append(per_head)
    return kept
