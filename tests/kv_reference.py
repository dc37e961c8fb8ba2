"""A plain implementation of the block-scaled KV cache for the tests, on the CPU: loops over sequences, blocks and heads.
Codes and scales by the definition's IEEE fp32 divisions (numpy), everything behind them in 64 bits."""
import numpy as np
import torch

FORMATS = {"i8": (torch.int8, 127.0), "e4m3": (torch.float8_e4m3fn, 448.0)}


def encode(x, s, fmt):
    """Codes (as bytes) of fp32 values x at an fp32 scale s; 0 at a scale that is not a number."""
    if not np.isfinite(s):
        return np.zeros(x.shape, np.uint8)
    y = (x.astype(np.float32) / np.float32(s)).astype(np.float32)
    dtype, most = FORMATS[fmt]
    y = torch.from_numpy(np.clip(np.rint(y) if fmt == "i8" else y, -most, most).astype(np.float32))
    return y.to(dtype).view(torch.uint8).numpy()


def decode(codes, fmt):
    return torch.from_numpy(codes.copy()).view(FORMATS[fmt][0]).float().numpy()


def write(codes, scale, table, x, kv_len, new_len, fmt):
    """codes [n, H, block, Dh] bytes and scale [n, H] fp32 are updated; x [B, S, H, Dh] fp32; table [B, max_blocks]."""
    n, H, block, Dh = codes.shape
    B, S = x.shape[:2]
    most = np.float32(FORMATS[fmt][1])
    for b in range(B):
        new = S if new_len is None else int(min(max(new_len[b], 0), S))
        origin = int(kv_len[b]) - new
        begin, end = max(origin, 0), min(int(kv_len[b]), table.shape[1] * block)
        for j in range(begin // block, -(-end // block) if end > begin else 0):
            blk = int(table[b, j])
            if not 0 <= blk < n:
                continue
            lo, hi = max(begin, j * block), min(end, (j + 1) * block)
            r0 = lo - j * block
            for h in range(H):
                rows = x[b, lo - origin:hi - origin, h].astype(np.float32)
                top = np.max(np.abs(rows))                                # (NaN wins)
                old = np.float32(scale[blk, h]) if r0 else np.float32(0)
                s = np.float32(np.nan)
                if np.isfinite(top) and not np.isnan(old):
                    s = max(old, np.float32(top / most), np.float32(2.0 ** -64))
                if r0 and not s == old:
                    c = decode(codes[blk, h, :r0], fmt)
                    codes[blk, h, :r0] = encode((c * old).astype(np.float32) if np.isfinite(s) else np.zeros_like(c), s, fmt)
                codes[blk, h, r0:r0 + hi - lo] = encode(np.where(np.isfinite(rows), rows, 0), s, fmt)
                scale[blk, h] = s


def rows_of(codes, scale, table, b, n, fmt):
    """Positions 0 .. n - 1 of sequence b in 64 bits, [n, H, Dh]; and the scale of each, [n, H], -1 where there is no block."""
    blocks, H, block, Dh = codes.shape
    out, scales = np.zeros((n, H, Dh)), np.full((n, H), -1.0)
    for j in range(-(-n // block)):
        blk, hi = int(table[b, j]), min(n, (j + 1) * block)
        if 0 <= blk < blocks:
            v = decode(codes[blk], fmt).astype(np.float64) * scale[blk].astype(np.float64)[:, None, None]
            out[j * block:hi] = v.transpose(1, 0, 2)[:hi - j * block]
            scales[j * block:hi] = scale[blk]
    return out, scales


def attend(q, ks, vs, v_scale, scale, causal, n):
    """q [S, Hq, Dh] (64 bits) of one sequence, the last n of whose keys are this call's: (out, sum p |v|, the largest sum |q k| |scale|
    of a row, the number of keys seen times the largest p v_scale).  Rows from n on, and those that see no key, are 0."""
    S, Hq, Dh = q.shape
    L, H, _ = ks.shape
    G = Hq // H
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    size, peak = np.zeros((S, Hq, 1)), np.zeros((S, Hq, 1))
    for i in range(min(S, n)):
        lim = min(L, max(0, i + 1 + L - n)) if causal else L
        vis = np.flatnonzero(v_scale[:lim, 0] >= 0)
        if not len(vis):
            continue
        for h in range(H):
            k, v, qq = ks[vis, h], vs[vis, h], q[i, h * G:(h + 1) * G]
            a = qq @ k.T * scale
            p = np.exp(a - a.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            out[i, h * G:(h + 1) * G], mag[i, h * G:(h + 1) * G] = p @ v, p @ np.abs(v)
            peak[i, h * G:(h + 1) * G, 0] = len(vis) * (p * v_scale[vis, h]).max(1)
            size[i, h * G:(h + 1) * G, 0] = (np.abs(qq) @ np.abs(k).T).max(1) * abs(scale)
    return out, mag, size, peak
