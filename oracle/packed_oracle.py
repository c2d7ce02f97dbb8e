"""Oracle of the operators over packed batches: numpy, 64 bits, written from their definitions.

Test infrastructure only, like stack_oracle: requests one by one, heads one by one, no shared code
with the library."""
import numpy as np


def batch_plan(lens, cached, free, table, max_tokens, block_size):
    """(cu, kv_len, slots, table, info) of spk_batch_plan."""
    lens, cached, table = list(map(int, lens)), list(map(int, cached)), np.array(table, np.int32)
    n, width = table.shape
    good = [max(v, 0) for v in lens]
    had = [max(v, 0) for v in cached]
    need = [-(-(c + v) // block_size) - -(-c // block_size) for c, v in zip(had, good)]
    why = (1 if sum(good) > max_tokens else 0) | (2 if sum(need) > len(free) else 0)
    for v, c in zip(lens, cached):
        why |= 8 if v < 0 or c < 0 else 4 if v + c > width * block_size else 0
    info = np.array([sum(good), sum(need), max(good), why], np.int32)
    slots = np.full(max_tokens, -1, np.int32)
    if why:
        return np.zeros(n + 1, np.int32), np.array(cached, np.int32), slots, table, info
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    taken = 0
    for r in range(n):
        held = -(-cached[r] // block_size)
        for j in range(need[r]):
            table[r, held + j] = free[taken]
            taken += 1
        for i in range(lens[r]):
            p = cached[r] + i
            slots[cu[r] + i] = table[r, p // block_size] * block_size + p % block_size
    return cu, (np.array(cached) + np.array(lens)).astype(np.int32), slots, table, info


def _softmax_parts(q, k, causal):
    """scores, their log-sum-exp, probabilities of one head of one request"""
    s = q @ k.T / np.sqrt(q.shape[1])
    if causal:
        s = np.where(np.tril(np.ones(s.shape, bool)), s, -np.inf)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    total = e.sum(-1, keepdims=True)
    return s, (m + np.log(total))[:, 0], e / total


def attention_packed(qkv, cu, hq, hkv, hd, causal):
    """o [T, hq, hd], lse [hq, T], and sum_j p_ij |v_j| [T, hq, hd]; rows of no request: 0.  qkv float64 [T, (hq + 2 hkv) * hd]."""
    T, g = qkv.shape[0], hq // hkv
    x = qkv.reshape(T, hq + 2 * hkv, hd)
    o, lse, weight = np.zeros((T, hq, hd)), np.zeros((hq, T)), np.zeros((T, hq, hd))
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(hq if b > a else 0):
            v = x[a:b, hq + hkv + h // g]
            _, lse[h, a:b], p = _softmax_parts(x[a:b, h], x[a:b, hq + h // g], causal)
            o[a:b, h], weight[a:b, h] = p @ v, p @ np.abs(v)
    return o, lse, weight


def attention_packed_bwd(qkv, cu, o, do, lse, hq, hkv, hd, causal):
    """dqkv [T, hq + 2 hkv, hd] from the forward's o and lse as they are given, the same sums over absolute values of what the
    kernels round to 16 bits (dS against q and k, P against dO), and over those of all that enters dS."""
    T, g, f = qkv.shape[0], hq // hkv, 1 / np.sqrt(hd)
    x, o, do = qkv.reshape(T, hq + 2 * hkv, hd), o.reshape(T, hq, hd), do.reshape(T, hq, hd)
    dx, rounded, entering = np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape)
    for a, b in zip(cu[:-1], cu[1:]):
        for h in range(hq if b > a else 0):
            ik, iv = hq + h // g, hq + hkv + h // g
            q, k, v, d = x[a:b, h], x[a:b, ik], x[a:b, iv], do[a:b, h]
            s, _, _ = _softmax_parts(q, k, causal)
            p = np.exp(s - lse[h, a:b, None])
            dp, delta = d @ v.T, (d * o[a:b, h]).sum(-1, keepdims=True)
            ds, big = p * (dp - delta) * f, p * (np.abs(d) @ np.abs(v).T + (np.abs(d) * np.abs(o[a:b, h])).sum(-1, keepdims=True)) * f
            dx[a:b, h] = ds @ k
            dx[a:b, ik] += ds.T @ q
            dx[a:b, iv] += p.T @ d
            rounded[a:b, h] = np.abs(ds) @ np.abs(k)
            rounded[a:b, ik] += np.abs(ds).T @ np.abs(q)
            rounded[a:b, iv] += p.T @ np.abs(d)
            entering[a:b, h] = big @ np.abs(k)
            entering[a:b, ik] += big.T @ np.abs(q)
            entering[a:b, iv] += p.T @ np.abs(d)
    return dx, rounded, entering


# ---- 8 bits ----------------------------------------------------------------------------------------

def e4m3_values():
    """What the 256 codes stand for: sign, 4 exponent bits (bias 7), 3 bits of mantissa, no infinities."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = (np.nan if c & 127 == 127 else x) * (-1 if c & 128 else 1)
    return v


E4M3 = e4m3_values()


def to_e4m3(x):
    """Codes of the nearest values, ties to the even code; not finite: NaN with its sign.  |x| <= 448."""
    x = np.asarray(x, np.float64)
    pos = E4M3[:127]
    a = np.where(np.isfinite(x), np.abs(x), 0)
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    up = a - pos[lo], pos[hi] - a
    code = np.where((up[0] > up[1]) | ((up[0] == up[1]) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def block_scale(x):
    """The smallest 2^e, e >= -126, with every finite |x| <= 448 * 2^e."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    e = -126
    while 448 * 2.0 ** e < top:
        e += 1
    return 2.0 ** e


def kv8_append(qkv, slots, k8, v8, scales, block_size, hq, hkv, hd):
    """k8 uint8 [blocks, hkv, bs, hd], v8 uint8 [blocks, hkv, hd, bs], scales [blocks, hkv, 2] afterwards (copies)."""
    k8, v8, scales = k8.copy(), v8.copy(), scales.astype(np.float64)
    x = qkv.reshape(qkv.shape[0], hq + 2 * hkv, hd)
    T, limit = len(slots), k8.shape[0] * block_size
    t = 0
    while t < T:
        s = int(slots[t])
        m = 1
        if 0 <= s < limit:
            b, off = divmod(s, block_size)
            while t + m < T and slots[t + m] == s + m and off + m < block_size:
                m += 1
            for h in range(hkv):
                for which, pool in ((0, k8[b, h]), (1, v8[b, h].T)):          # [bs, hd], views
                    new = x[t:t + m, hq + which * hkv + h]
                    scale = block_scale(new)
                    if off:
                        old = scales[b, h, which]
                        scale = max(scale, old)
                        if scale > old:
                            pool[:off] = to_e4m3(E4M3[pool[:off]] * (old / scale))
                    pool[off:off + m] = to_e4m3(new / scale)
                    scales[b, h, which] = scale
        t += m
    return k8, v8, scales


def kv8_attention(q, k8, v8, scales, table, kv_len, block_size):
    """o [B, hq, hd] and sum p |v|; q float64 [B, hq, hd]."""
    B, hq, hd = q.shape
    blocks, hkv = k8.shape[:2]
    o, weight = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        pos = np.arange(min(max(int(kv_len[b]), 0), table.shape[1] * block_size))
        blk = table[b, pos // block_size]
        pos, blk = pos[(blk >= 0) & (blk < blocks)] % block_size, blk[(blk >= 0) & (blk < blocks)]
        for h in range(hq if pos.size else 0):
            kh = h // (hq // hkv)
            k = E4M3[k8[blk, kh, pos]] * scales[blk, kh, 0][:, None]
            v = E4M3[v8[blk, kh, :, pos]] * scales[blk, kh, 1][:, None]
            s = k @ q[b, h] / np.sqrt(hd)
            p = np.exp(s - s.max())
            p /= p.sum()
            o[b, h], weight[b, h] = p @ v, p @ np.abs(v)
    return o, weight
