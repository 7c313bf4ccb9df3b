"""The e4m3 cache's format in 64 bits on the host, for the tests: quantisation from its definition,
the values of a cache, and plain writers and readers token by token."""
import numpy as np
import torch

D = 128
E_MIN, E_MAX = -117, 119


def quantise(x):
    """(values y = code, exponent e) of float64 rows [..., 128]: the least e with max|x| <= 448 * 2^e
    in [-117, 119], y = x / 2^e on the e4m3 grid (ties to even), within +-448."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    e = np.full(top.shape, E_MAX, np.int64)
    for c in range(E_MAX - 1, E_MIN - 1, -1):
        e = np.where(top <= np.ldexp(448.0, c), c, e)
    y = np.clip(x * np.ldexp(1.0, -e)[..., None], -448, 448)
    _, k = np.frexp(y)                       # |y| in [2^(k-1), 2^k)
    grid = np.ldexp(1.0, np.maximum(k - 1, -6) - 3)
    return np.rint(y / grid) * grid, e


def values(codes, exps):
    """float64 [P][Hkv][ps][128] (K's or V's) from float8 codes and exps[..., j, :] bytes."""
    c = codes.detach().cpu().to(torch.float32).numpy().astype(np.float64)
    e = exps.detach().cpu().numpy().astype(np.int64)
    return np.ldexp(c, e.reshape(e.shape[0], e.shape[1], -1)[..., None] - 127)


def both_values(k8, v8, exps):
    return values(k8, exps[:, :, :, 0]), values(v8, exps[:, :, :, 1])


def row_of(L, n, cu, b, pos):
    return cu[b] + pos - (L - n)


def append(k, v, cu, bt, lens, ps, kv, vv, meta, mean=False):
    """Plain writer: float64 rows k, v [T][Hkv][128] into value arrays kv, vv [P][Hkv][ps][128] and
    float64 landmarks (in place), sequence by sequence and token by token."""
    P, M = kv.shape[0], bt.shape[1]
    for b, L in enumerate(int(x) for x in lens):
        n = max(0, int(cu[b + 1]) - int(cu[b]))
        if L < 1 or L > M * ps:
            continue
        for pos in range(max(0, L - n), L):
            phys, slot = int(bt[b, pos // ps]), pos % ps
            if not 0 <= phys < P:
                continue
            r = cu[b] + pos - (L - n)
            for rows, arr in ((k, kv), (v, vv)):
                y, e = quantise(rows[r])
                arr[phys, :, slot] = np.ldexp(y, e[:, None])
            key = kv[phys, :, slot]
            if mean:
                old = 0.0 if slot == 0 else meta[phys]
                meta[phys] = np.float32(np.float32(old) + key.astype(np.float32))
            elif slot == 0:
                meta[phys, :, 0], meta[phys, :, 1] = key, key
            else:
                meta[phys, :, 0] = np.minimum(meta[phys, :, 0], key)
                meta[phys, :, 1] = np.maximum(meta[phys, :, 1], key)


def read(kv, cu, bt, lens, T, fill):
    """Plain reader of one value array: float64 [T][Hkv][128], rows that no sequence has = fill."""
    P, Hkv, ps, _ = kv.shape
    out = np.full((T, Hkv, D), float(fill))
    for b, L in enumerate(int(x) for x in lens):
        n = max(0, int(cu[b + 1]) - int(cu[b]))
        for pos in range(L - n, L):
            phys = int(bt[b, pos // ps]) if 0 <= pos < bt.shape[1] * ps else -1
            out[cu[b] + pos - (L - n)] = kv[phys, :, pos % ps] if 0 <= phys < P else 0.0
    return out
