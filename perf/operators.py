"""The measured work of the operators that run a quantized network: products of matrices held in 8-bit floating point with a
scale for each block of 128, and attention over a cache of keys and values held in 4 bits.

  quantize   a matrix of activations or weights into 8-bit floating point blocks
  codes      a layer's 4-bit codes, as `fobq_quantize_layer` returns them, as such a matrix
  matmul     the product of activations and a weight matrix, both in blocks
  append     new keys and values into the 4-bit cache, and read back from it as the values they stand for
  attention  attention of packed query rows over that cache

With `own` false everything is elementary torch in 32 bits; with `own` true it is the calls a user makes.
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 128
TINY = 2.0 ** -126
TOP = {"e4m3": 448.0, "e5m2": 57344.0}
FLOAT8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
FLOAT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one decoding step of eight sequences: the input of a layer of 4608 columns; the launch is all there is
        dict(name="quantize_tokens", kind="quantize", rows=8, cols=4608, src="bf16", fmt="e4m3", per=1),
        # a large weight matrix, once per model, 128 x 128 blocks
        dict(name="quantize_weights", kind="quantize", rows=8192, cols=8192, src="f32", fmt="e4m3", per=128),
        # the 3x3 convolution 256 -> 256 of a ResNet-50 at 4 bits, one grid per row
        dict(name="codes_conv3x3", kind="codes", rows=256, cols=2304, bits=4, group=0),
        # the widest quantized layer: 3 bits in groups of 128 columns
        dict(name="codes_wide_g128", kind="codes", rows=2048, cols=4608, bits=3, group=128),
        # one token through a large layer: the weights are read once
        dict(name="matmul_token", kind="matmul", m=1, n=8192, k=8192, a="e4m3", b="e4m3", per=128, dst="bf16"),
        # a ragged batch through a quantized layer of 1000 outputs, a scale per weight row and block, results in 32 bits
        dict(name="matmul_ragged", kind="matmul", m=777, n=1000, k=2304, a="e4m3", b="e4m3", per=1, dst="f32"),
        # a long prompt through a large layer
        dict(name="matmul_prompt", kind="matmul", m=8192, n=8192, k=8192, a="e4m3", b="e4m3", per=128, dst="bf16"),
        # one decoding step of 64 sequences
        dict(name="append_step", kind="append", seqs=64, new=1, length=4096, heads=8, dim=128, page=64, src="bf16"),
        # four prompts of about 4096 tokens
        dict(name="append_prompts", kind="append", seqs=4, new=4096, length=4096, heads=8, dim=128, page=64, src="bf16"),
        # one decoding step of two short sequences: latency
        dict(name="decode_short", kind="attention", seqs=2, new=1, length=600, heads=8, group=4, dim=128, page=16, src="bf16", causal=True, window=0),
        # one decoding step of 32 sequences with long caches, one slot of the batch idle
        dict(name="decode_long", kind="attention", seqs=32, new=1, length=16384, heads=8, group=4, dim=128, page=64, src="bf16", causal=True, window=0),
        # three prompts of about 2048 tokens behind caches that hold as much already
        dict(name="prompts", kind="attention", seqs=3, new=2048, length=5000, heads=8, group=4, dim=128, page=64, src="bf16", causal=True, window=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "codes", "matmul", "matmul", "matmul", "append", "attention", "attention", "attention"])
    if kind == "quantize":
        cols = _log(rng, 32, 16384)
        return dict(kind=kind, rows=_log(rng, 1, max(2, min(32768, 6.4e7 / cols))), cols=cols, src=rng.choice(list(FLOAT)), fmt=rng.choice(["e4m3", "e4m3", "e5m2"]),
                    per=rng.choice([1, 1, 128]))
    if kind == "codes":
        cols, group = _log(rng, 64, 4608), rng.choice([0, 128, 256])
        cols = cols if not group else max(group, cols // group * group)
        return dict(kind=kind, rows=_log(rng, 16, 2048), cols=cols, bits=rng.choice([2, 3, 4]), group=group)
    if kind == "matmul":
        n, k = _log(rng, 64, 8192), _log(rng, 64, 8192)
        m = rng.choice([_log(rng, 1, 64), _log(rng, 16, 8192)])
        return dict(kind=kind, m=m, n=n, k=k, a=rng.choice(["e4m3", "e4m3", "e5m2"]), b=rng.choice(["e4m3", "e4m3", "e5m2"]), per=rng.choice([1, 128, 128]),
                    dst=rng.choice(["bf16", "bf16", "f16", "f32"]))
    dim = rng.choice([64, 128, 128, 256])
    heads, page, src = rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 256]), rng.choice(["bf16", "bf16", "f16"])
    if kind == "append":
        seqs = _log(rng, 1, 128)
        new = rng.choice([1, _log(rng, 1, max(2, 16384 // seqs))])
        return dict(kind=kind, seqs=seqs, new=new, length=new - 1 + _log(rng, 1, 4096), heads=heads, dim=dim, page=page, src=src)
    group = rng.choice([1, 2, 4, 4, 7, 8])
    new = rng.choice([1, 1, _log(rng, 2, 8), _log(rng, 16, 2048)])
    length = new - 1 + _log(rng, 1, 16384 if new < 16 else 4096)
    seqs = _log(rng, 1, max(2, min(64, 5.0e5 / (length * heads / 8 * dim / 128), 6.0e8 / (new * heads * group * length * dim / 128))))
    return dict(kind=kind, seqs=seqs, new=new, length=length, heads=heads, group=group, dim=dim, page=page, src=src, causal=rng.random() < 0.85,
                window=rng.choice([0, 0, 0, _log(rng, 1, 2048)]))


# ---- sequences --------------------------------------------------------------------------------------------------
def _sequences(case):
    """(tokens in the cache, new tokens) of every sequence of a case: ragged, the first one the longest; in a step of single
    tokens over four sequences or more the last slot of the batch is idle (nothing in its cache)."""
    r = random.Random("%(seqs)d %(new)d %(length)d %(page)d" % case)
    got = []
    for i in range(case["seqs"]):
        new = case["new"] if i == 0 or case["new"] == 1 else r.randint(max(1, case["new"] // 2), case["new"])
        top = case["length"]
        got.append((top if i == 0 else r.randint(max(new, top // 3), top), new))
    if case["kind"] == "attention" and case["new"] == 1 and case["seqs"] >= 4:
        got[-1] = (0, 1)
    return got


def _cdiv(a, b):
    return -(-a // b)


def _visible(case, length, new, i):
    """The range of tokens that new token i of a sequence sees."""
    end = length - new + i + 1 if case["causal"] else length
    start = max(0, end - case["window"]) if case["window"] else 0
    return start, max(start, end)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _normal(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _activations(g, rows, cols, dtype):
    """Gaussian rows, a few columns of which are an order of magnitude larger, as a network's hidden states have them."""
    x = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.float32)
    big = torch.rand((cols,), generator=g, device="cuda") < 0.01
    return (x * torch.where(big, 10.0, 1.0)).to(dtype)


def _pad16(t):
    """The same 8-bit matrix with rows a multiple of 16 bytes apart."""
    rows, cols = t.shape
    at = torch.zeros((rows, _cdiv(cols, 16) * 16), dtype=torch.uint8, device=t.device)
    at[:, :cols] = t.view(torch.uint8)
    return at.view(t.dtype)[:, :cols]


def _pages(case, g):
    """A cache with pages in random order, and what says which sequence has which."""
    seqs, page = _sequences(case), case["page"]
    width = max(1, max(_cdiv(n, page) for n, _ in seqs))
    count = sum(_cdiv(n, page) for n, _ in seqs) + 3
    order = torch.randperm(count, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(seqs), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, (n, _) in enumerate(seqs):
        have = _cdiv(n, page)
        table[i, :have] = order[at:at + have]
        at += have
    starts = [0]
    for _, new in seqs:
        starts.append(starts[-1] + new)
    dims = (count, case["heads"], page)
    cache = {n: torch.zeros(dims + (case["dim"] // 2,), dtype=torch.uint8, device="cuda") for n in ("k_codes", "v_codes")}
    cache.update({n: torch.zeros(dims, dtype=torch.int32, device="cuda") for n in ("k_grids", "v_grids")})
    return {"cache": cache, "table": table, "lengths": torch.tensor([n for n, _ in seqs], dtype=torch.int32, device="cuda"),
            "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"), "rows": starts[-1], "longest": max(n for n, _ in seqs)}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind, state = case["kind"], {"case": case}
    if kind == "quantize":
        state["x"] = _activations(g, case["rows"], case["cols"], FLOAT[case["src"]])
    elif kind == "codes":
        rows, cols, top = case["rows"], case["cols"], 2 ** case["bits"] - 1
        groups = cols // case["group"] if case["group"] else 1
        state["codes"] = (_normal(g, (rows, cols)) * (top / 6.0) + top / 2.0).round_().clamp_(0, top).to(torch.uint8)
        state["scales"] = torch.rand((rows, groups), generator=g, device="cuda") * 0.01 + 0.005
        state["zeros"] = (_normal(g, (rows, groups)) * 0.6 + top / 2.0).round_().clamp_(0, top)
    elif kind == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        state["a"] = [_pad16(t) if i == 0 else t for i, t in enumerate(_blocks(_activations(g, m, k, torch.float32), case["a"], 1))]
        state["b"] = [_pad16(t) if i == 0 else t for i, t in enumerate(_blocks(_normal(g, (n, k)) * math.sqrt(2.0 / k), case["b"], case["per"]))]
    else:
        state.update(_pages(case, g))
        heads, dim, rows, dtype = case["heads"], case["dim"], state["rows"], FLOAT[case["src"]]
        if kind == "append":
            # keys and values are parts of the rows that one product made
            both = _activations(g, rows, 2 * heads * dim, dtype).view(rows, 2 * heads, dim)
            state["k"], state["v"] = both[:, :heads], both[:, heads:]
        else:
            state["q"] = _normal(g, (rows, heads * case["group"], dim), dtype)
            for n in ("k", "v"):
                pages = state["cache"][n + "_codes"].shape[0]
                step = max(1, (1 << 26) // (heads * case["page"] * dim))
                for lo in range(0, pages, step):
                    part = slice(lo, min(pages, lo + step))
                    shape = (part.stop - lo, heads, case["page"], dim)
                    state["cache"][n + "_codes"][part], state["cache"][n + "_grids"][part] = _grid16(_normal(g, shape, dtype))
            state["scale"] = dim ** -0.5
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _blocks(x, fmt, per):
    """A matrix as 8-bit values and the scales of its blocks of `per` rows and 128 columns, block columns first."""
    rows, cols = x.shape
    br, bc = _cdiv(rows, per), _cdiv(cols, BLOCK)
    p = torch.nn.functional.pad(x.float(), (0, bc * BLOCK - cols, 0, br * per - rows)).view(br, per, bc, BLOCK)
    most = p.abs().amax((1, 3))
    scale = torch.where(most.isfinite(), (most / TOP[fmt]).clamp(min=TINY), math.nan)
    v = (p / scale[:, None, :, None]).clamp(-TOP[fmt], TOP[fmt]).to(FLOAT8[fmt]).view(br * per, bc * BLOCK)
    return v[:rows, :cols], scale.t().contiguous()


def _unblock(v, scales, per):
    rows, cols = v.shape
    s = scales.t().repeat_interleave(per, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]
    return v.float() * s


def _grid16(x):
    """Rows of 16 levels: two codes a byte, the even channel in the low half, and a word that holds the scale (bf16) above the
    zero point.  The quotients are divisions by tensors, which round once: values of few bits often lie on the border of two levels."""
    x = x.float()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    bits = ((hi - lo) / torch.full_like(hi, 15.0)).view(torch.int32)
    scale = ((bits + 0xFFFF) & -65536).view(torch.float32).clamp(min=TINY)
    zero = (-lo / scale).round().clamp(0.0, 15.0)
    codes = ((x / scale[..., None]).round() + zero[..., None]).clamp(0.0, 15.0).to(torch.uint8)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), scale.view(torch.int32) | zero.to(torch.int32)


def _values(codes, grids):
    """What such rows stand for."""
    scale, zero = (grids & -65536).view(torch.float32), (grids & 15).float()
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
    return (c - zero[..., None]) * scale[..., None]


def _slots(state):
    """(page, slot) of every packed row."""
    page, starts = state["case"]["page"], state["starts"].long()
    row = torch.arange(state["rows"], device="cuda")
    seq = torch.searchsorted(starts, row, right=True) - 1
    at = state["lengths"].long()[seq] - starts[seq + 1] + row
    return state["table"][seq, at // page].long(), at % page


def _append(state):
    at, cache = _slots(state), state["cache"]
    for n in ("k", "v"):
        codes, grids = _grid16(state[n])
        cache[n + "_codes"][at[0], :, at[1]] = codes
        cache[n + "_grids"][at[0], :, at[1]] = grids
    return [_values(cache[n + "_codes"][at[0], :, at[1]], cache[n + "_grids"][at[0], :, at[1]]).to(state[n].dtype) for n in ("k", "v")]


def _attention(state):
    case, cache, q = state["case"], state["cache"], state["q"]
    heads, group, dim, seqs, new = case["heads"], case["group"], case["dim"], case["seqs"], case["new"]
    table, lengths, starts = state["table"].long().clamp(min=0), state["lengths"].long(), state["starts"].long()
    k, v = (_values(cache[n + "_codes"][table].transpose(1, 2), cache[n + "_grids"][table].transpose(1, 2)).reshape(seqs, heads, -1, dim) for n in ("k", "v"))
    have = starts[1:] - starts[:-1]
    i = torch.arange(new, device="cuda")
    at = starts[:-1, None] + torch.minimum(i[None], have[:, None] - 1)
    rows = q[at].float().view(seqs, new, heads, group, dim).permute(0, 2, 3, 1, 4).reshape(seqs, heads, group * new, dim)
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()).view(seqs, heads, group, new, -1).mul_(state["scale"])
    t = torch.arange(score.shape[-1], device="cuda")
    end = (lengths - have)[:, None] + i[None] + 1 if case["causal"] else lengths[:, None].expand(seqs, new)
    seen = (t < end[..., None]) & (t < lengths[:, None, None])
    if case["window"]:
        seen &= t >= end[..., None] - case["window"]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = score.sum(-1, keepdim=True)
    out = torch.matmul(score.view(seqs, heads, group * new, -1), v).view(seqs, heads, group, new, dim) / torch.where(total > 0, total, 1.0)
    mine = (i[None] < have[:, None])
    return out.permute(0, 3, 1, 2, 4)[mine].reshape(-1, heads * group, dim).to(q.dtype)


def _plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "quantize":
        return list(_blocks(state["x"], case["fmt"], case["per"]))
    if kind == "codes":
        groups, rep = state["scales"].shape[1], case["group"] // BLOCK if case["group"] else _cdiv(case["cols"], BLOCK)
        zeros = state["zeros"].repeat_interleave(case["cols"] // groups, 1)
        return [(state["codes"].float() - zeros).to(torch.float8_e4m3fn), state["scales"].repeat_interleave(rep, 1).t().contiguous()]
    if kind == "matmul":
        return torch.matmul(_unblock(*state["a"], 1), _unblock(*state["b"], case["per"]).t()).to(FLOAT[case["dst"]])
    return _append(state) if kind == "append" else _attention(state)


# ---- the framework's calls ------------------------------------------------------------------------------------------
_handle = []


def _context():
    """The context that a program keeps for as long as it runs."""
    import paper_2509_05576_amd as fobq
    if not _handle:
        _handle.append(fobq.Ctx(0))
    return fobq, _handle[0]


def _calls(state):
    fobq, ctx = _context()
    case = state["case"]
    kind = case["kind"]
    if kind == "quantize":
        m = ctx.fp8_quantize(state["x"], FLOAT8[case["fmt"]], rows_per_scale=case["per"])
        return [m.values, m.scales]
    if kind == "codes":
        m = ctx.fp8_from_codes(state["codes"], state["scales"], state["zeros"], bits=case["bits"])
        return [m.values, m.scales]
    if kind == "matmul":
        return ctx.fp8_matmul(fobq.Fp8Matrix(*state["a"], 1), fobq.Fp8Matrix(*state["b"], case["per"]), FLOAT[case["dst"]])
    cache = fobq.Kv4Cache(**state["cache"])
    batch = fobq.Kv4Batch(state["table"], state["lengths"], state["starts"])
    if kind == "append":
        ctx.kv4_append(cache, batch, state["k"], state["v"])
        return list(ctx.kv4_read(cache, batch, state["rows"], state["k"].dtype))
    return ctx.kv4_attention(cache, batch, state["q"], scale=state["scale"], causal=case["causal"], window=case["window"], max_length=state["longest"])


def run(state):
    return _calls(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (BYTES[case["src"]] + 1) + 4 * _cdiv(case["rows"], case["per"]) * _cdiv(case["cols"], BLOCK), "flops": 2 * n}
    if kind == "codes":
        n, groups = case["rows"] * case["cols"], case["cols"] // case["group"] if case["group"] else 1
        return {"bytes": 2 * n + 8 * case["rows"] * groups + 4 * case["rows"] * _cdiv(case["cols"], BLOCK), "flops": n}
    if kind == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + 4 * _cdiv(k, BLOCK) * (m + _cdiv(n, case["per"])) + m * n * BYTES[case["dst"]], "flops": 2 * m * n * k}
    size, heads, dim, seqs = BYTES[case["src"]], case["heads"], case["dim"], _sequences(case)
    rows = sum(new for _, new in seqs)
    if kind == "append":
        # in: keys and values; out: two cache rows per token and head, which are read again, and the values read
        return {"bytes": rows * heads * (4 * dim * size + 2 * (dim + 8)), "flops": 12 * rows * heads * dim}
    pairs, tokens = 0, 0
    for length, new in seqs:
        spans = [_visible(case, length, new, i) for i in range(new)]
        pairs += sum(b - a for a, b in spans)
        tokens += max(b for _, b in spans) - min(a for a, _ in spans)
    return {"bytes": tokens * heads * (dim + 8) + 2 * rows * heads * case["group"] * dim * size, "flops": 4 * pairs * heads * case["group"] * dim}


# ---- the same in 64 bits ------------------------------------------------------------------------------------------------
def _power2(e):
    """2^e in 64 bits, from its bits: exact on every device."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _round8(x, fmt):
    """Nearest value of an 8-bit type, ties to the even one, in 64 bits."""
    keep, low = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = torch.frexp(x)
    step = _power2((e - 1).clamp(min=low) - keep)
    return (x / step).round() * step


def _exact_blocks(x, fmt, per):
    rows, cols = x.shape
    v, scales = torch.empty((rows, cols), dtype=torch.float64, device=x.device), []
    for c in range(0, cols, BLOCK):
        part = x[:, c:c + BLOCK].double()
        most = part.abs().amax(1)
        most = torch.stack([p.max() for p in most.split(per)]) if per > 1 else most
        scales.append((most / TOP[fmt]).clamp(min=TINY))
        v[:, c:c + BLOCK] = _round8(part / scales[-1].repeat_interleave(per)[:rows, None], fmt).clamp(-TOP[fmt], TOP[fmt])
    return v, torch.stack(scales)


def _exact_rows(x):
    """Rows rounded to their 16 levels and back, in 64 bits."""
    x = x.double()
    lo, hi = x.amin(-1, keepdim=True).clamp(max=0.0), x.amax(-1, keepdim=True).clamp(min=0.0)
    _, e = torch.frexp((hi - lo) / 15.0)
    step = _power2(e - 8)
    scale = (torch.ceil((hi - lo) / (15.0 * step)) * step).clamp(min=TINY)
    zero = torch.round(-lo / scale)
    return ((torch.round(x / scale) + zero).clamp(0.0, 15.0) - zero) * scale


def _exact_cached(cache, name, pages, length):
    """heads x length x dim of one sequence, from its pages."""
    codes, word = cache[name + "_codes"][pages], cache[name + "_grids"][pages]
    low, high = (codes % 16).double(), torch.div(codes, 16, rounding_mode="floor").double()
    level = torch.stack((low, high), -1).flatten(-2) - (word % 16).double()[..., None]
    level *= (word - word % 65536).view(torch.float32).double()[..., None]
    return level.transpose(0, 1).flatten(1, 2)[:, :length]


def exact(case, seed):
    state, kind = prepare(case, seed), case["kind"]
    if kind == "quantize":
        return list(_exact_blocks(state["x"], case["fmt"], case["per"]))
    if kind == "codes":
        wide = case["group"] or case["cols"]
        v = torch.cat([c.double() - state["zeros"][:, i:i + 1].double() for i, c in enumerate(state["codes"].split(wide, 1))], 1)
        at = [c // wide for c in range(0, case["cols"], BLOCK)]
        return [v, state["scales"].double()[:, at].t().contiguous()]
    if kind == "matmul":
        (a, sa), (b, sb), out = state["a"], state["b"], 0.0
        for i, c in enumerate(range(0, case["k"], BLOCK)):
            left = a[:, c:c + BLOCK].double() * sa[i].double()[:, None]
            right = b[:, c:c + BLOCK].double() * sb[i].double().repeat_interleave(case["per"])[:case["n"], None]
            out = out + left @ right.t().contiguous()
        return out
    if kind == "append":
        return [_exact_rows(state["k"]), _exact_rows(state["v"])]
    heads, group, dim = case["heads"], case["group"], case["dim"]
    out, at = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda"), 0
    for s, (length, new) in enumerate(_sequences(case)):
        if length:
            pages = state["table"][s, :_cdiv(length, case["page"])].long()
            k, v = (_exact_cached(state["cache"], n, pages, length) for n in ("k", "v"))
            spans = torch.tensor([_visible(case, length, new, i) for i in range(new)], device="cuda")
            t = torch.arange(length, device="cuda")
            hide = ((t < spans[:, :1]) | (t >= spans[:, 1:])).repeat_interleave(group, 0)
            q = state["q"][at:at + new].double().view(new, heads, group, dim)
            for h in range(heads):
                p = (q[:, h].reshape(new * group, dim) @ k[h].t().contiguous()) * state["scale"]
                p = torch.softmax(p.masked_fill_(hide, -math.inf), 1).nan_to_num_(0.0)
                out[at:at + new].view(new, heads, group, dim)[:, h] = (p @ v[h]).view(new, group, dim)
        at += new
    return out
