"""Plain numpy forms, in 64 bits, of the operators for drafted tokens, and the error that the kernel's arithmetic allows."""
import numpy as np

from oracle import cronus_oracle as orc

BLOCK = 16


def random_tree_mask(rng, n, words, density=None):
    """Mask rows of n tokens: a random tree (density None), or random bits, the row itself not always among them."""
    rows = np.zeros((n, n), dtype=bool)
    if density is None:
        for i in range(n):
            if i:
                rows[i] = rows[int(rng.integers(0, i))]
            rows[i, i] = True
    else:
        rows = rng.random((n, n)) < density
    return rows, pack_mask(rows, words)


def pack_mask(rows, words):
    n = rows.shape[0]
    bits = np.zeros((n, words * 64), dtype=np.uint8)
    bits[:, :rows.shape[1]] = rows
    return np.packbits(bits, axis=1, bitorder="little").view(np.uint64).reshape(n, words).view(np.int64)


def attention(q, k, v, seen, sm_scale, accumulated=None):
    """q [n][Hq][D], k, v [kv][Hkv][D] (float64), seen [n][kv] bool: (result, bound on the kernel's error), both [n][Hq][D].

    The kernel's own errors, relative to a weight w_j of the row: the numerator is rounded to bf16, half a step or 2^-8, and the
    sum that divides it adds the rounded ones; the score's error e_s = scale * sum |q k| (D + 8) 2^-24 (products of bf16 are exact, their sum and the
    factor are rounded in fp32) and a few ulp of exp2.  With relative errors of at most e of every weight the result moves by at most
    e / (1 - e) * sum_j w_j |V_j - out| <= e (1 + 2^-6) (A + |out|), A = sum_j w_j |V_j|.  Sums over the keys in fp32 (the row's
    result, twice where it is rescaled or merged): (kv + 32) 2^-23 A.  The result is rounded to bf16: 2^-8 of it."""
    n, hq, d = q.shape
    hkv = k.shape[1]
    out, bound = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    if not k.shape[0]:
        return out, bound
    for h in range(hq):
        g = h // (hq // hkv)
        with np.errstate(invalid="ignore", over="ignore"):
            x = np.where(seen, (q[:, h] @ k[:, g].T) * sm_scale, -np.inf)
            mag = (np.abs(q[:, h]) @ np.abs(k[:, g]).T * sm_scale).max(axis=1, where=seen, initial=0.0)
            top = x.max(axis=1, initial=-np.inf)
            w = np.exp(x - np.where(np.isneginf(top), 0.0, top)[:, None])
            total = w.sum(axis=1)
            w = w / np.where(total == 0, 1.0, total)[:, None]
            vz = np.where(np.isfinite(v[:, g]), v[:, g], 0.0)
            out[:, h], a = w @ vz, w @ np.abs(vz)
            for j in np.flatnonzero(~np.isfinite(v[:, g]).all(axis=1)):  # reach the rows that see them
                out[:, h] += np.where(seen[:, j, None], w[:, j, None] * np.where(np.isfinite(v[j, g]), 0.0, v[j, g]), 0.0)
            e = 2.0 ** -8 + mag * (d + 8) * 2.0 ** -24 + 2.0 ** -20
            bound[:, h] = (e * (1 + 2.0 ** -6))[:, None] * (a + np.abs(w @ vz)) + (k.shape[0] + 32) * 2.0 ** -23 * a + 2.0 ** -8 * np.abs(w @ vz)
        nothing = ~seen.any(axis=1)
        out[nothing, h] = 0.0
        hidden_nan = np.isnan(x).any(axis=1, where=seen) | ((total == 0) & ~nothing)
        out[hidden_nan, h] = np.nan
    return out, bound


def seen_of(prefix, n, rows=None):
    """Visible keys of n drafted tokens behind `prefix` cached ones; rows None: a chain."""
    tail = np.tril(np.ones((n, n), dtype=bool)) if rows is None else rows
    return np.concatenate([np.ones((n, prefix), dtype=bool), tail], axis=1)


def tables(kv, new, held, table, free, count, capacity, max_tokens):
    """cronus_build_tables: dict of all that it writes (slots: of the tokens alone)."""
    kv, new, held = (np.asarray(x, dtype=np.int64) for x in (kv, new, held))
    n, width = table.shape
    table, free = table.copy(), list(free[:count])
    rest = {"cu_tokens": np.zeros(n + 1, int), "cu_blocks": np.zeros(n + 1, int), "start": kv, "held": held, "count": count}
    bad = next((s for s in range(n) if kv[s] < 0 or new[s] < -1 or held[s] < 0 or held[s] > width or -(-kv[s] // BLOCK) > held[s] or
                kv[s] + max(new[s], 0) > width * BLOCK), -1)
    if bad >= 0:
        return {**rest, "status": 1, "bad": bad}
    back = [int(b) for s in range(n) if new[s] == -1 for b in table[s, :held[s]]]
    if not 0 <= count <= capacity or count + len(back) > capacity:
        return {**rest, "status": 1, "bad": -1}
    need = np.where(new < 0, 0, np.maximum(0, -(-(kv + np.maximum(new, 0)) // BLOCK) - held))
    add = np.maximum(new, 0)
    if need.sum() > count + len(back):
        return {**rest, "status": 2, "asked": (int(add.sum()), int(need.sum()))}
    if add.sum() > max_tokens:
        return {**rest, "status": 3, "asked": (int(add.sum()), int(need.sum()))}
    free += back
    pushed = list(free)
    start, slots = np.where(new < 0, 0, kv), []
    for s in range(n):
        for i in range(int(need[s])):
            table[s, held[s] + i] = free.pop()
        slots += [int(table[s, p // BLOCK]) * BLOCK + p % BLOCK for p in range(int(start[s]), int(start[s] + add[s]))]
    return {"status": 0, "bad": -1, "asked": (int(add.sum()), int(need.sum())), "table": table, "pushed": pushed, "count": len(free),
            "held": np.where(new < 0, 0, held) + need, "start": start, "cu_tokens": np.concatenate([[0], np.cumsum(add)]),
            "cu_blocks": np.concatenate([[0], np.cumsum(need)]), "slots": np.array(slots, dtype=np.int64)}


def path_in_effect(path, length, n):
    """How many entries of a path count."""
    m, before = 0, -1
    for a in path[:max(0, min(int(length), len(path)))]:
        if not before < a < n:
            break
        m, before = m + 1, a
    return m


def k_view(pool, hkv, d):
    return pool.reshape(-1, hkv, d // 8, BLOCK, 8)


def v_view(pool, hkv, d):
    return pool.reshape(-1, hkv, 2, d, 8)


def commit(k_pool, v_pool, hkv, d, start, cu, paths, path_lens, table):
    """Moves rows in the pools (in place); returns the new lengths."""
    k, v = k_view(k_pool, hkv, d), v_view(v_pool, hkv, d)
    lens = np.array(start, dtype=np.int64)
    for s in range(len(start)):
        n, at = int(cu[s + 1] - cu[s]), int(start[s])
        if at < 0 or n <= 0 or at + n > table.shape[1] * BLOCK:
            continue
        m = path_in_effect(paths[s], path_lens[s], n)
        place = lambda p: (int(table[s, p // BLOCK]), p % BLOCK)  # noqa: E731
        rows = [(k[b, :, :, t].copy(), v[b, :, t // 8, :, t % 8].copy()) for b, t in (place(at + int(a)) for a in paths[s][:m])]
        for i, (kr, vr) in enumerate(rows):
            b, t = place(at + i)
            k[b, :, :, t], v[b, :, t // 8, :, t % 8] = kr, vr
        lens[s] = at + m
    return lens


def read_rows(k_pool, v_pool, hkv, d, table, positions):
    """(k, v) bits [n][Hkv][D] of one sequence's positions."""
    k, v = k_view(k_pool, hkv, d), v_view(v_pool, hkv, d)
    pos = np.asarray(positions)
    b, t = table[pos // BLOCK], pos % BLOCK
    return k[b, :, :, t].reshape(len(pos), hkv, d), v[b, :, t // 8, :, t % 8].reshape(len(pos), hkv, d)


def write_rows(k_pool, v_pool, hkv, d, table, positions, k_rows, v_rows):
    k, v = k_view(k_pool, hkv, d), v_view(v_pool, hkv, d)
    pos = np.asarray(positions)
    b, t = table[pos // BLOCK], pos % BLOCK
    k[b, :, :, t] = k_rows.reshape(len(pos), hkv, d // 8, 8)
    v[b, :, t // 8, :, t % 8] = v_rows


def values(bits, scale=None):
    """float64 of cached bits [n][Hkv][D]: bf16 patterns, or e4m3 codes times the KV head's scale."""
    if scale is None:
        return orc.bf16_bits_to_f64(bits)
    with np.errstate(invalid="ignore"):
        return E4M3[bits] * np.asarray(scale, dtype=np.float32).astype(np.float64)[None, :, None]


E4M3 = orc.fp8_e4m3_decode(np.arange(256, dtype=np.uint8))
