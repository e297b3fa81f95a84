"""Plain 64-bit statement of the 8-bit cache for the tests: quantising, the block layout, attention over the cached values.
Shares no code with the library."""
from __future__ import annotations

import numpy as np

from paper_2402_01869_amd import binding as B
from paper_2402_01869_amd import workloads as W

BLOCK = 16
FORMATS = {"e4m3": B.IC_DTYPE_E4M3, "int8": B.IC_DTYPE_INT8}
TOP = {"e4m3": 448.0, "int8": 127.0}


def code_values(fmt: str) -> np.ndarray:
    """What the 256 codes stand for (before the scale)."""
    c = np.arange(256)
    if fmt == "int8":
        return np.where(c < 128, c, c - 256).astype(np.float64)
    sign, ex, m = c >> 7, (c >> 3) & 15, c & 7
    mag = np.where(ex == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (ex.astype(np.float64) - 10))
    mag[(ex == 15) & (m == 7)] = np.nan
    return np.where(sign == 1, -mag, mag)


def quantise(bits: np.ndarray, fmt: str):
    """bf16 bit patterns [..., D] -> codes uint8 [..., D], scale bytes uint8 [...]; nearest code, ties to the even one."""
    x = W.bf16_bits_to_f64(bits).reshape(-1, bits.shape[-1])
    table = code_values(fmt)
    order = np.array([c for c in range(128) if not np.isnan(table[c]) and table[c] <= TOP[fmt]])  # ascending magnitudes
    mags = table[order]
    codes, scales = np.zeros(x.shape, dtype=np.uint8), np.zeros(x.shape[0], dtype=np.uint8)
    for i, v in enumerate(x):
        if not np.isfinite(v).all():
            scales[i] = 255
            continue
        a = np.abs(v).max()
        e = -100
        if a > TOP[fmt] * 2.0 ** -100:
            e = int(np.ceil(np.log2(a) - np.log2(TOP[fmt]))) - 2  # well below, then the definition itself
            while a > TOP[fmt] * 2.0 ** e:
                e += 1
            e = max(e, -100)
        y = np.abs(v) / 2.0 ** e
        hi = np.minimum(np.searchsorted(mags, y), len(mags) - 1)
        lo = np.maximum(hi - 1, 0)
        up, down = mags[hi] - y, y - mags[lo]
        pick = np.where(up < down, hi, np.where(down < up, lo, np.where(order[hi] % 2 == 0, hi, lo)))
        c = order[pick]
        codes[i] = np.where(np.signbit(v), (c + 128 if fmt == "e4m3" else (256 - c) % 256), c).astype(np.uint8)
        scales[i] = e + 127
    return codes.reshape(bits.shape), scales.reshape(bits.shape[:-1])


def values(codes: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    v = code_values(fmt)[codes] * np.exp2(scales.astype(np.float64) - 127.0)[..., None]
    v[scales == 255] = np.nan
    return v


def split(pool: np.ndarray, Hkv: int, D: int):
    """Views of a pool's bytes [blocks][block bytes]: codes [blocks][2][Hkv][16][D], scale bytes [blocks][Hkv][2][16]."""
    at = 2 * Hkv * BLOCK * D
    return pool[:, :at].reshape(-1, 2, Hkv, BLOCK, D), pool[:, at:at + 2 * Hkv * BLOCK].reshape(-1, Hkv, 2, BLOCK)


def empty_pool(num_blocks: int, Hkv: int, D: int, fill: int = 0xFF) -> np.ndarray:
    """0xff: NaN codes of e4m3, and the scale byte of a NaN vector."""
    return np.full((num_blocks, B.block_bytes(Hkv, D, BLOCK, B.IC_DTYPE_INT8)), fill, dtype=np.uint8)


def write(pool: np.ndarray, batch, k_bits, v_bits, fmt: str) -> None:
    """kv_write_span, on the host."""
    Hkv, D = k_bits.shape[1:]
    codes, scales = split(pool, Hkv, D)
    for i, new in enumerate((k_bits, v_bits)):
        c, s = quantise(new, fmt)
        for seq in range(batch.num_seqs):
            for r in range(int(batch.q_len[seq])):
                t = int(batch.ctx_len[seq] - batch.q_len[seq]) + r
                b, slot, row = int(batch.block_tables[seq, t // BLOCK]), t % BLOCK, int(batch.q_start[seq]) + r
                codes[b, i, :, slot] = c[row]
                scales[b, :, i, slot] = s[row]


def random_pool(batch, Hkv: int, D: int, fmt: str, rng, spread: int = 3) -> np.ndarray:
    """Every live slot random codes with scales of a few sizes (values of magnitude about 1), everything else 0xff."""
    pool = empty_pool(batch.pool_blocks, Hkv, D)
    codes, scales = split(pool, Hkv, D)
    for s in range(batch.num_seqs):
        ctx = int(batch.ctx_len[s])
        for j, b in enumerate(batch.block_tables[s, :-(-ctx // BLOCK)]):
            n = min(BLOCK, ctx - j * BLOCK)
            x = rng.standard_normal((2, Hkv, n, D)) * TOP[fmt] / 4
            if fmt == "int8":
                c = np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
            else:
                c = _near_e4m3(x)
            codes[b, :, :, :n] = c
            scales[b, :, :, :n] = rng.integers(-spread, 2, (Hkv, 2, n)) + 127 - (7 if fmt == "e4m3" else 5)
    return pool


def _near_e4m3(x):
    t = code_values("e4m3")[:127]
    c = np.minimum(np.searchsorted(t, np.abs(x)), 126).astype(np.uint8)
    return np.where(x < 0, c | 128, c).astype(np.uint8)


def context(pool, batch, s, Hkv, D, fmt):
    """K, V [ctx][Hkv][D] in 64 bits of one sequence."""
    codes, scales = split(pool, Hkv, D)
    t = np.arange(int(batch.ctx_len[s]))
    b, slot = batch.block_tables[s, t // BLOCK], t % BLOCK
    return tuple(values(codes[b, i][t, :, slot], scales[b][t, :, i, slot], fmt) for i in (0, 1))


def attention(pool, batch, q_bits, Hkv, fmt):
    """(out, dev) [rows][H][D] in 64 bits: softmax(scale q K^T) V of every row over the keys up to its position, and the mean
    distance of a value from the result under the same weights, which is what an error of the weights is multiplied by."""
    q = W.bf16_bits_to_f64(q_bits)
    _, H, D = q.shape
    out, dev = np.full(q.shape, np.nan), np.zeros(q.shape)
    for s in range(batch.num_seqs):
        K, V = context(pool, batch, s, Hkv, D, fmt)
        c, n, r0 = int(batch.ctx_len[s]), int(batch.q_len[s]), int(batch.q_start[s])
        for h in range(H):
            k, v = K[:, h // (H // Hkv)], V[:, h // (H // Hkv)]
            w = q[r0:r0 + n, h] @ k.T * float(np.float32(batch.scale))
            for i in range(n):
                p = w[i, :c - n + i + 1]
                p = np.exp(p - p.max())
                p /= p.sum()
                out[r0 + i, h] = p @ v[:len(p)]
                dev[r0 + i, h] = p @ np.abs(v[:len(p)] - out[r0 + i, h])
    return out, dev
