"""Plain 64-bit forms of the 8-bit block matrices and of the 4-bit cache with its attention, on the CPU, from their definitions, with
the bounds that the kernels' arithmetic gives."""
import ctypes
import math

import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.float8_e5m2: 57344.0}
KEEP_LOW = {torch.float8_e4m3fn: (3, -6), torch.float8_e5m2: (2, -14)}
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}   # half a step
U = 2.0 ** -24
TINY = 2.0 ** -126


def power2(e):
    return torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e)


def step8(x, fmt):
    """The distance of 8-bit values around x."""
    keep, low = KEEP_LOW[fmt]
    _, e = torch.frexp(x)
    return power2((e - 1).clamp(min=low) - keep)


def round8(x, fmt):
    s = step8(x, fmt)
    return (x / s).round() * s


def blocks(rows, cols, per):
    for j in range(0, cols, 128):
        for i in range(0, rows, per):
            yield i // per, j // 128, slice(i, min(rows, i + per)), slice(j, min(cols, j + 128))


def quantize(x, fmt, per):
    """(quotients, scales): what the 8-bit values are the nearest ones to."""
    x = x.double()
    rows, cols = x.shape
    q, scales = torch.empty_like(x), torch.empty((-(-cols // 128), -(-rows // per)), dtype=torch.float64)
    for bi, bj, r, c in blocks(rows, cols, per):
        most = x[r, c].abs().max()
        if not bool(torch.isfinite(x[r, c]).all()):
            scales[bj, bi], q[r, c] = math.nan, math.nan
            continue
        scales[bj, bi] = max(float(most) / TOP[fmt], TINY)
        q[r, c] = x[r, c] * TOP[fmt] / most if float(most) / TOP[fmt] > TINY else x[r, c] / TINY
    return q, scales


def expand(values, scales, per):
    s = scales.double().t().repeat_interleave(per, 0)[:values.shape[0]].repeat_interleave(128, 1)[:, :values.shape[1]]
    return values.double() * s


def matmul(a, b, dtype):
    """(product, bound) of expanded matrices: fp32 sums of k products in any order, two fp32 operations a block of 128 on top, one
    rounding to `dtype` (half the smallest step where the result is denormal).  A result in 16 bits may come from the 8-bit matrix
    instruction, which adds eight neighbouring products to 13 bits below the largest."""
    y, weight = a @ b.t(), a.abs() @ b.abs().t()
    k = a.shape[1]
    bound = (k + 3 * (-(-k // 128)) + 4) * U * weight + HALF[dtype] * y.abs() * 1.01 + torch.finfo(dtype).smallest_normal * HALF[dtype]
    if dtype != torch.float32:
        eights = lambda x: torch.nn.functional.pad(x.abs(), (0, -k % 8)).unflatten(1, (-1, 8)).amax(2)  # noqa: E731
        bound += 8 * 2.0 ** -13 * (eights(a) @ eights(b).t())
    return y, bound


# ---- the 4-bit cache -----------------------------------------------------------------------------------------------
def grid(x):
    """(codes, scale, zero) of rows of finite values."""
    x = x.double()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    _, e = torch.frexp((hi - lo) / 15.0)
    step = power2(e - 8)
    scale = (torch.ceil((hi - lo) / (15.0 * step)) * step).clamp(min=TINY)
    zero = torch.round(-lo / scale)
    return (torch.round(x / scale[..., None]) + zero[..., None]).clamp(0.0, 15.0), scale, zero


def unpack(codes, grids):
    """(code - zero, scale) of cache rows."""
    g = grids.to(torch.int64) & 0xFFFFFFFF
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).double()
    scale = ((g >> 16) << 16).to(torch.int64)
    scale = torch.where(scale >= 1 << 31, scale - (1 << 32), scale).to(torch.int32).view(torch.float32).double()
    return c - (g & 15).double()[..., None], scale


def attention(q, k, v, scale, spans, dtype):
    """One sequence and head of the cache.  q: rows x dim; k, v: (code - zero, scale) of its tokens; spans: per row the tokens seen.
    Returns (out, lse, bound of out, bound of lse)."""
    (kc, ks), (vc, vs) = k, v
    rows, dim = q.shape
    out, lse = torch.zeros((rows, dim), dtype=torch.float64), torch.full((rows,), -math.inf, dtype=torch.float64)
    bound, lbound = torch.zeros_like(out), torch.zeros((rows,), dtype=torch.float64)
    for i, (a, b) in enumerate(spans):
        if b <= a:
            continue
        x = q[i].double()
        s = (kc[a:b] @ x) * ks[a:b] * scale
        top = s.max()
        p = (s - top).exp()
        total = p.sum()
        val = vc[a:b] * vs[a:b, None]
        out[i], lse[i] = p @ val / total, top + total.log()
        # scores: bf16 keys enter as 128 + code, at most 143, and 128 + zero is taken off again: sums of dim terms in fp32, then
        # three roundings; the exponential to 2 units of fp32 and its argument's rounding
        ds = ((dim + 8) * U * 2 * 143 * x.abs().sum() * ks[a:b] * abs(scale) + 4 * U * s.abs()).max() + 8 * U * (top - s.min()).clamp(max=160) + 8 * U
        n = b - a
        # weights times scales in fp16, 2^-11 each, below 2^-14 of the row's largest to 2^-25 of it
        bound[i] = ((2.0 ** -11 * 1.01 + 2 * ds + (n + 64) * U) * (p @ val.abs()) + n * 2.0 ** -25 * (p * vs[a:b]).max() * 15) / total
        bound[i] += HALF[dtype] * out[i].abs() * 1.01 + 1e-37
        lbound[i] = 2 * ds + (n + 64) * U + 4 * U * lse[i].abs()
    return out, lse, bound, lbound


# ---- the structs of include/fobq.h, for calls with fields of their own ----------------------------------------------
def _struct(name, pointers, longs, ints, floats=(), last=()):
    fields = [(n, ctypes.c_void_p) for n in pointers] + [(n, ctypes.c_int64) for n in longs] + [(n, ctypes.c_int32) for n in ints]
    return type(name, (ctypes.Structure,), {"_fields_": fields + [(n, ctypes.c_float) for n in floats] + [(n, ctypes.c_int32) for n in last]})


Fp8Struct = _struct("Fp8Struct", ("values", "scales"), ("rows", "cols", "ld", "ld_scales"), ("rows_per_scale", "format"))
CacheStruct = _struct("CacheStruct", ("k_codes", "v_codes", "k_grids", "v_grids"), ("pages",), ("page_size", "heads", "head_dim", "reserved"))
BatchStruct = _struct("BatchStruct", ("table", "lengths", "starts"), ("rows", "table_ld"), ("n_seqs", "max_pages"))
QueryStruct = _struct("QueryStruct", ("Q", "out", "lse"), ("q_row", "q_head", "out_row", "out_head", "max_length"), ("type", "group", "causal", "window"),
                      ("scale",), ("reserved",))
