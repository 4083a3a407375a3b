"""The operators in plain 64-bit arithmetic, for the tests: numpy, one row or one sequence at a time, from the definitions in include/sdlm.h."""
import numpy as np

PAGE = 16


def sample_row(z, t, k, p, m, u):
    """(id, probability); z, t, p, m, u as doubles of the values that the operator is given."""
    z = np.where(np.isnan(z), -np.inf, np.asarray(z, dtype=np.float64))
    top = z.max()
    if top == -np.inf:
        return -1, 0.0
    order = np.lexsort((np.arange(z.size), -z))
    if not t > 0:
        return int(order[0]), 1.0
    order = order[z[order] > -np.inf]
    with np.errstate(invalid="ignore"):
        w = np.where(z[order] == top, 1.0, np.exp((z[order] - top) / t))
    if k > 0:
        order, w = order[:k], w[:k]
    keep = len(w)
    if p < 1:
        before = np.cumsum(w) - w
        keep = min(keep, max(1, int(np.sum(before < p * w.sum()))))
    if m > 0:
        keep = min(keep, max(1, int(np.sum(w >= min(m, 1.0)))))
    w = w[:keep]
    cum = np.cumsum(w)
    at = min(int(np.sum(cum <= min(max(u, 0.0), 1.0) * cum[-1])), int(np.sum(w > 0)) - 1)
    return int(order[at]), float(w[at] / cum[-1])


def k_index(slot, i):
    return i // 8 * 128 + slot * 8 + i % 8


def v_index(slot, i):
    return (i // 16 * 4 + slot // 4) * 64 + i % 16 * 4 + slot % 4


def rows_at(layer_tiles, tiles, slots, h, d):
    """K and V rows [n, d] of kv head h at the given tiles and slots; layer_tiles [tiles, kv heads, 2, 16 d]."""
    i = np.arange(d)[None, :]
    s = np.asarray(slots)[:, None]
    t = layer_tiles[np.asarray(tiles, dtype=np.int64), h]
    n = np.arange(len(slots))[:, None]
    return t[:, 0][n, k_index(s, i)], t[:, 1][n, v_index(s, i)]


def tree_attention(layer_tiles, q, table, lens, offs, seen, node_table, node_base):
    """layer_tiles [tiles, kv heads, 2, 16 d] and q [rows, heads, d] as float64; seen: bool [rows, most nodes].  Rows of no sequence stay NaN."""
    hkv, d = layer_tiles.shape[1], layer_tiles.shape[3] // PAGE
    G = q.shape[1] // hkv
    out = np.full(q.shape, np.nan)
    for b, n in enumerate(lens):
        r0, r1 = offs[b], offs[b + 1]
        T = r1 - r0
        pos = np.concatenate([np.arange(n), node_base[b] + np.arange(T)]).astype(np.int64)
        tabs = np.concatenate([table[b][pos[:n] // PAGE], node_table[b][pos[n:] // PAGE]])
        for h in range(hkv):
            K, V = rows_at(layer_tiles, tabs, pos % PAGE, h, d)
            for r in range(r0, r1):
                see = np.concatenate([np.ones(n, bool), seen[r, :T]])
                for g in range(h * G, h * G + G):
                    if not see.any():
                        out[r, g] = 0.0
                        continue
                    s = K[see] @ q[r, g] / np.sqrt(d)
                    w = np.exp(s - s.max())
                    out[r, g] = (w / w.sum()) @ V[see]
    return out


def fork(cache, parent, share):
    """cache: dict of table [S, pages], lens, held, refs and pool ([layers, tiles, ...], copied in place); returns the new cache or a status."""
    S, pps = cache["table"].shape
    n_pages = len(cache["refs"])
    if any(p < -1 or p >= S for p in parent):
        return 2
    own, plan = {}, []
    for b, p in enumerate(parent):       # who keeps a parent's own pages
        if p >= 0:
            own[p] = p if p < len(parent) and parent[p] == p else own.get(p, b)
    refs = [0] * n_pages
    for b, p in enumerate(parent):
        held = cache["held"][p] if p >= 0 else 0
        keep = held if p >= 0 and own[p] == b else (cache["lens"][p] // PAGE if share and p >= 0 else 0)
        plan.append((held, keep))
        for j in range(keep):
            refs[cache["table"][p][j]] += 1
    free = [i for i in range(n_pages) if refs[i] == 0]
    need = sum(h - k for h, k in plan)
    if need > len(free):
        return 1
    new = {"table": np.full((S, pps), -1, np.int32), "lens": np.zeros(S, np.int32), "held": np.zeros(S, np.int32), "pool": cache["pool"].copy()}
    for b, p in enumerate(parent):
        held, keep = plan[b]
        if p < 0:
            continue
        new["lens"][b], new["held"][b] = cache["lens"][p], held
        for j in range(held):
            page = cache["table"][p][j]
            if j >= keep:
                fresh = free.pop(0)
                refs[fresh] = 1
                if j * PAGE < cache["lens"][p]:
                    new["pool"][:, fresh] = cache["pool"][:, page]
                page = fresh
            new["table"][b, j] = page
    new["refs"] = np.array(refs, np.int32)
    new["free"] = np.array(free + [-1] * (n_pages - len(free)), np.int32)
    new["n_free"] = len(free)
    return new


def compact(pool, table, lens, path, path_len, node_table, node_base):
    """pool [layers, tiles, kv heads, 2, 16 d]; returns the pool after the moves."""
    old, out = pool, pool.copy()
    d = pool.shape[4] // PAGE
    i = np.arange(d)
    for b in range(len(path)):
        for m in range(path_len[b]):
            src, dst = node_base[b] + path[b][m], lens[b] + m
            ts, td = node_table[b][src // PAGE], table[b][dst // PAGE]
            for which, index in ((0, k_index), (1, v_index)):
                out[:, td, :, which, index(dst % PAGE, i)] = old[:, ts, :, which, index(src % PAGE, i)]
    return out
