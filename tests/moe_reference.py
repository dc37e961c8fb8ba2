"""The operators of a mixture-of-experts MLP by their definition, in loops and 64 bits."""
import numpy as np
import torch

import oracle as O
from paper_2310_17723_amd import binding as HB

EPS = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}              # half a step of a 16-bit result, relative
ODT = {torch.bfloat16: O.BF16, torch.float16: O.F16}


def route(logits, k, renorm):
    """(expert, weight in 64 bits, slot, row_token, offsets, the largest |l - m| of a finite logit) of a float32 array [T, E]."""
    T, E = logits.shape
    l = np.where(np.isnan(logits), -np.inf, np.minimum(logits.astype(np.float64), np.finfo(np.float32).max))
    expert, slot, weight = np.full((T, k), -1), np.full((T, k), -1), np.zeros((T, k))
    for t in range(T):
        order = sorted(range(E), key=lambda e: (-l[t, e], e))
        chosen = [e for e in order[:k] if l[t, e] > -np.inf]
        if not chosen:
            continue
        p = np.exp(l[t] - l[t].max())
        total = p[chosen].sum() if renorm else p.sum()
        expert[t, :len(chosen)] = chosen
        weight[t, :len(chosen)] = p[chosen] / total
    rows = [[(t, j) for t in range(T) for j in range(k) if expert[t, j] == e] for e in range(E)]
    offsets, token = [0], np.full(T * k, -1)
    for e in range(E):
        for i, (t, j) in enumerate(rows[e]):
            slot[t, j], token[offsets[-1] + i] = offsets[-1] + i, t
        offsets.append(offsets[-1] + len(rows[e]))
    return expert, weight, slot, token, np.array(offsets)


def clean_offsets(offsets, R):
    """The rows that each expert has, whatever the offsets are: the running maximum within [0, R]."""
    return np.maximum.accumulate(np.clip(offsets, 0, R))


def sources(row_index, R, MA):
    return np.arange(R) if row_index is None else np.clip(row_index, 0, MA - 1)


def product8(fmt, A, W, offsets, row_index, a_row_scale, b_col_scale, bias, epi, out_col_scale, c_dt):
    """{expert: (rows, the oracle's result)} for 8-bit operands."""
    E = W.shape[0]
    R = A.shape[0] if row_index is None else len(row_index)
    at, src = clean_offsets(offsets, R), sources(row_index, R, A.shape[0])
    fn = O.int8_gemm if fmt == "i8" else O.fp8_gemm
    pick = lambda v, e: None if v is None else v[e]  # noqa: E731
    out = {}
    for e in range(E):
        if at[e] < at[e + 1]:
            rows = src[at[e]:at[e + 1]]
            out[e] = (slice(at[e], at[e + 1]), fn(A[rows], W[e], a_row_scale=None if a_row_scale is None else a_row_scale[rows], b_col_scale=b_col_scale[e],
                                                  bias=pick(bias, e), epi=epi, out_col_scale=pick(out_col_scale, e), c_dt=c_dt))
    return out


def gelu(x):
    return 0.5 * x * (1 + torch.erf(x * 0.5 ** 0.5))


def product_hp(A, W, offsets, row_index, bias, act):
    """{expert: (rows, result, sum |a w|)} in 64 bits, on the CPU."""
    R = A.shape[0] if row_index is None else len(row_index)
    at, src = clean_offsets(offsets, R), sources(row_index, R, A.shape[0])
    out = {}
    for e in range(W.shape[0]):
        if at[e] < at[e + 1]:
            a, w = A[torch.as_tensor(src[at[e]:at[e + 1]])].double(), W[e].double()
            y = a @ w.t()
            if bias is not None:
                y = y + bias[e].double()
            out[e] = (slice(at[e], at[e + 1]), gelu(y) if act else y, a.abs() @ w.abs().t())
    return out


def combine(y, slot, weight, residual):
    """(out, sum of |terms|) in 64 bits."""
    T, k = slot.shape
    out = np.zeros((T, y.shape[1])) if residual is None else residual.astype(np.float64)
    mag = np.abs(out)
    for t in range(T):
        for j in range(k):
            if 0 <= slot[t, j] < y.shape[0]:
                out[t] = out[t] + float(weight[t, j]) * y[slot[t, j]].astype(np.float64)
                mag[t] = mag[t] + np.abs(float(weight[t, j]) * y[slot[t, j]].astype(np.float64))
    return out, mag


EPI_OF = {"dequant": HB.EPI_DEQUANT, "gelu": HB.EPI_DEQUANT_GELU, "requant": HB.EPI_REQUANT, "gelu_requant": HB.EPI_GELU_REQUANT}
