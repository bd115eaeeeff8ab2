"""Microscaled 4-bit codes and what is computed from them, on the CPU in 64 bits: the definitions, for the tests."""
import numpy as np
import torch

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def blocks_of(n):
    return (n + 31) // 32


def panels_of(n):
    return (n + 255) // 256


def mix(x):
    x = np.asarray(x, np.uint64)
    low = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x85EBCA6B)) & low
    x = x ^ (x >> np.uint64(13))
    x = (x * np.uint64(0xC2B2AE35)) & low
    return x ^ (x >> np.uint64(16))


def draws(index, seed):
    low = np.uint64(0xFFFFFFFF)
    lo, hi = np.uint64(seed & 0xFFFFFFFF), np.uint64((seed >> 32) & 0xFFFFFFFF)
    kx = mix(lo ^ mix((hi + np.uint64(0x9E3779B9)) & low))
    ka = mix((kx + np.uint64(0x9E3779B9)) & low)
    return mix(((np.asarray(index, np.uint64) & low ^ kx) + ka) & low) >> np.uint64(8)


def quantise(x, u=None):
    """Rows of x (numpy, finite or not) in blocks of 32: (codes 0 .. 15 (rows, 32 blocks), bytes (rows, blocks)).  u: 24-bit draws of x's shape."""
    x = np.asarray(x, np.float64)
    rows, n = x.shape
    k = blocks_of(n)
    v = np.zeros((rows, 32 * k))
    v[:, :n] = x
    v = v.reshape(rows, k, 32)
    with np.errstate(all="ignore"):
        m = np.abs(v).max(-1)
        ok = np.isfinite(m)
        safe = np.where(ok & (m > 0), m, 1.0)
        f, e = np.frexp(safe)                        # m = f 2^e, 1/2 <= f < 1: 6 = .75 2^3
        e = np.where(f <= 0.75, e - 3, e - 2)
        e = np.clip(np.where(ok & (m > 0), e, -127), -127, 127)
        a = np.where(ok[..., None], np.ldexp(np.abs(np.where(ok[..., None], v, 0)), -e[..., None]), 0.0)
    assert a.max(initial=0) <= 6
    if u is None:
        step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
        mag = np.searchsorted(LEVELS, np.rint(a / step) * step)
    else:
        uu = np.zeros((rows, 32 * k), np.int64)
        uu[:, :n] = np.asarray(u, np.int64) >> 2
        low = np.clip(np.searchsorted(LEVELS, a, side="right") - 1, 0, 6)
        place = np.floor((a - LEVELS[low]) / (LEVELS[low + 1] - LEVELS[low]) * 2.0**22)
        mag = low + (place + uu.reshape(rows, k, 32) >= 2.0**22)
    code = mag + 8 * (np.signbit(v) & ok[..., None])
    return code.reshape(rows, 32 * k), np.where(ok, e + 127, 255)


def stands_for(code, byte, n):
    """What codes and bytes stand for, (rows, n)."""
    v = np.where(code & 8, -1.0, 1.0) * LEVELS[code & 7]
    with np.errstate(all="ignore"):
        s = np.where(byte == 255, np.nan, np.ldexp(1.0, np.asarray(byte, np.int64) - 127))
    return (v.reshape(*byte.shape, 32) * s[..., None]).reshape(code.shape[0], -1)[:, :n]


def rounded(x, u=None):
    """x as its codes hold it."""
    return stands_for(*quantise(x, u), np.asarray(x).shape[1])


def packed(code):
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)


def unpacked(q):
    q = np.asarray(q)
    out = np.empty(q.shape[:-1] + (2 * q.shape[-1],), np.int64)
    out[..., 0::2], out[..., 1::2] = q & 15, q >> 4
    return out


def in_panels(byte, n):
    """Bytes (rows, blocks) as [panels][rows][8]."""
    out = np.zeros((panels_of(n) * 8, byte.shape[0]), np.uint8)
    out[:byte.shape[1]] = byte.T
    return np.ascontiguousarray(out.reshape(-1, 8, byte.shape[0]).transpose(0, 2, 1))


def cache_values(cache):
    """(keys, values) of a PagedCache4 as (pages, heads, page_size, dim), 64 bits."""
    out = []
    for q, s in ((cache.kq, cache.ks), (cache.vq, cache.vs)):
        q, s = q.cpu().numpy(), s.cpu().numpy()
        v = stands_for(unpacked(q.reshape(-1, q.shape[-1])), s.reshape(-1, s.shape[-1]), cache.dim)
        out.append(torch.from_numpy(v.reshape(q.shape[:3] + (cache.dim,))))
    return out
