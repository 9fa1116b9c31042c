"""The cache's operators in plain numpy, 64 bits, token by token: what the tests compare with.

Contents are kept by position ([request][kv head, token, channel] numbers and a
scale per page), so nothing here shares the library's byte order but
``key_bytes`` and ``value_bytes``, which say where a token's byte lies.
"""
import numpy as np

PAGE = 64
TOP = {0: 448.0, 1: 127.0}          # by ugbs_cache_type


def key_at(d):
    t, c = np.arange(PAGE)[:, None], np.arange(d)[None]
    return t // 16 * 16 * d + c // 64 * 1024 + c % 64 // 16 * 256 + t % 16 * 16 + c % 16


def value_at(d):
    t, c = np.arange(PAGE)[:, None], np.arange(d)[None]
    return t // 32 * 32 * d + c // 32 * 1024 + t % 16 // 4 * 256 + c % 16 * 16 + c % 32 // 16 * 8 + t % 32 // 16 * 4 + t % 4


def _e4m3_numbers():
    b = np.arange(256)
    e, m = b // 8 % 16, b % 8
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x = np.where((e == 15) & (m == 7), np.nan, x)
    return np.where(b > 127, -x, x)


NUMBERS = {0: _e4m3_numbers(), 1: np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)}


def nearest(x, dtype):
    """x to the nearest number of the type, ties to even."""
    if dtype == 1:
        return np.clip(np.rint(x), -127, 127)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.clip(np.rint(x / step) * step, -448, 448)


def scale_of(amax, dtype):
    s = 2.0 ** -100
    while amax > TOP[dtype] * s:
        s *= 2.0
    return s


def decode(cache, scales, dtype, d):
    """Raw cache [n_pages, Hkv, 2, 64 d] uint8 and scales -> keys, values [n_pages, Hkv, 64, d] in 64 bits."""
    k = NUMBERS[dtype][cache[:, :, 0][..., key_at(d)]] * scales[..., 0][..., None, None].astype(np.float64)
    v = NUMBERS[dtype][cache[:, :, 1][..., value_at(d)]] * scales[..., 1][..., None, None].astype(np.float64)
    return k, v


def encode(k, v, dtype):
    """Numbers (without scale) [n_pages, Hkv, 64, d] -> raw bytes [n_pages, Hkv, 2, 64 d]."""
    d = k.shape[-1]
    out = np.zeros(k.shape[:2] + (2, PAGE * d), np.uint8)
    for w, (x, at) in enumerate(((k, key_at(d)), (v, value_at(d)))):
        if dtype == 1:
            b = x.astype(np.int64).astype(np.int8).view(np.uint8)
        else:
            table = NUMBERS[0][:127]                                    # 0 .. 448, rising
            b = np.searchsorted(table, np.abs(x)).astype(np.uint8)
            b = b | np.where(np.signbit(x), 128, 0).astype(np.uint8)
        flat = out[:, :, w]
        flat[..., at] = b
    return out


def plan(ctx, new, stack, count, table, rows):
    """ugbs_cache_plan, request by request: (stack, table, kv, q, slots, left)."""
    B, mp = table.shape
    n_pages = len(stack)
    stack, table = list(map(int, stack)), table.copy()
    h = min(max(int(count), 0), n_pages)
    most = PAGE * mp
    asked = []
    for b in range(B):
        c, n = int(ctx[b]), int(new[b])
        sound = 0 <= c <= most
        c = min(max(c, 0), most)
        held = -(-c // PAGE)
        if sound and n == -1:
            for p in range(held):
                if h < n_pages:
                    stack[h] = int(table[b, p])
                    h += 1
            asked.append((c, 0, held, True))
        else:
            ok = sound and 0 <= n <= rows and c + n <= most
            asked.append((c, n if ok else 0, held, False))
    kv, q = np.zeros(B, np.int32), np.zeros(B, np.int32)
    slots = np.full((B, rows), -1, np.int32)
    wanted, left = 0, h
    for b, (c, n, held, gone) in enumerate(asked):
        need = -(-(c + n) // PAGE) - held
        start = wanted
        wanted += need
        if gone:
            continue
        kv[b] = c
        if need and wanted > h:
            continue
        for j in range(need):
            table[b, held + j] = stack[h - 1 - start - j]
        if need:
            left = h - wanted
        kv[b], q[b] = c + n, n
        for i in range(n):
            page = int(table[b, (c + i) // PAGE])
            if 0 <= page < n_pages:
                slots[b, i] = PAGE * page + (c + i) % PAGE
    return np.array(stack, np.int32), table, kv, q, slots, left


def store(K, V, slots, cache, scales, dtype):
    """ugbs_cache_store on copies of cache and scales; K, V [B, Hkv, rows, d] in 64 bits."""
    B, Hkv, rows, d = K.shape
    cache, scales = cache.copy(), scales.copy()
    where = (key_at(d), value_at(d))
    for b in range(B):
        i = 0
        while i < rows and slots[b, i] >= 0:
            page, t0 = divmod(int(slots[b, i]), PAGE)
            n = 1
            while i + n < rows and t0 + n < PAGE and slots[b, i + n] == slots[b, i] + n:
                n += 1
            for h in range(Hkv):
                for w, X in enumerate((K, V)):
                    x = X[b, h, i:i + n]
                    s = scale_of(np.abs(x).max(), dtype)
                    raw = cache[page, h, w]
                    if t0:
                        was = float(scales[page, h, w])
                        s = max(s, was)
                        if s > was:
                            old = nearest(NUMBERS[dtype][raw[where[w][:t0]]] * (was / s), dtype)
                            raw[where[w][:t0]] = _bytes(old, dtype)
                    raw[where[w][t0:t0 + n]] = _bytes(nearest(x / s, dtype), dtype)
                    scales[page, h, w] = s
            i += n
    return cache, scales


def _bytes(x, dtype):
    if dtype == 1:
        return x.astype(np.int64).astype(np.int8).view(np.uint8)
    return (np.searchsorted(NUMBERS[0][:127], np.abs(x)) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def attend(Q, k, v, there, kv, q, scale):
    """One request: Q [H, n, d]; k, v [Hkv, positions, d]; there [positions] (the position lies in a page);
    the q newest of kv tokens.  64 bits; rows without a key, and rows q and up, give 0.  Also the weighted
    sizes of the values and the largest sum |q k| scale of each row: (O, sizes [H, n, d], spread [H, n])."""
    H, n, d = Q.shape
    G = H // k.shape[0]
    out, sizes, spread = np.zeros((H, n, d)), np.zeros((H, n, d)), np.zeros((H, n))
    last = kv - q + np.arange(q)
    seen = there[None, :] & (np.arange(len(there))[None, :] <= last[:, None])
    rows = np.flatnonzero(seen.any(1))
    if not len(rows):
        return out, sizes, spread
    seen = seen[rows]
    for h in range(H):
        kk, vv = k[h // G], v[h // G]
        s = np.where(seen, (Q[h, rows] @ kk.T) * scale, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[h, rows] = p @ np.where(there[:, None], vv, 0)
        sizes[h, rows] = p @ np.abs(np.where(there[:, None], vv, 0))
        spread[h, rows] = np.where(seen, np.abs(Q[h, rows]) @ np.abs(kk).T, 0).max(1) * scale
    return out, sizes, spread
