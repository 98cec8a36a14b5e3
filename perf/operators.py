"""Cases of the rank-local half of an expert layer: the tokens' slots sorted by expert, the rows gathered into that
order and brought back, the quantisers, and the block-scaled 8-bit products of the experts.

A case is a dict of plain values.  `prepare` builds on the GPU what a program has in hand before the call, `run` makes
one pass (the plain form in elementary torch operations, or the framework's calls), and `exact` computes the same
outputs in 64 bits.  An 8-bit matrix is a float8_e4m3fn tensor whose rows are whole blocks of 128 (zeros past the end)
beside its scales, fp32 or float8_e8m0fnu (powers of two), whose rows hold a multiple of four blocks.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ESIZE = {"bf16": 2, "f32": 4}
F8 = torch.float8_e4m3fn
E8M0 = torch.float8_e8m0fnu
BLOCK = 128
F8_MAX = 448.0
SCALE_MIN = 2.0 ** -126


def listed():
    return [
        # Routing of one decode step of 64 tokens, top-8 of 256 experts, all of them here: bound by latency.
        dict(name="sort_decode", op="sort", tokens=64, topk=8, experts=256, parts=1),
        # Routing of a long prefill (an odd number of tokens) seen from one of 8 ranks, which holds 32 of the 256.
        dict(name="sort_prefill", op="sort", tokens=32771, topk=8, experts=256, parts=8),
        # The same decode step's rows into expert order, quantised on the way for the experts' first product.
        dict(name="gather_decode", op="gather", tokens=64, topk=8, experts=256, parts=1, hidden=7168, dtype="bf16",
             scale="e8m0"),
        # A training step's rows into expert order, kept in 16 bits; a width that is no multiple of 128.
        dict(name="gather_train", op="gather", tokens=4099, topk=4, experts=32, parts=1, hidden=2880, dtype="bf16",
             scale="none"),
        # The way back of a decode step, with the router's weights.
        dict(name="scatter_decode", op="scatter", tokens=64, topk=8, experts=256, parts=1, hidden=7168, dtype="bf16",
             weighted=True),
        # The gradient of the way back for 8 ranks' 512 tokens on one rank: rows and weights.
        dict(name="scatter_grad", op="scatter_grad", tokens=4096, topk=8, experts=256, parts=8, hidden=7168,
             dtype="bf16"),
        # Activations between an expert's two products, quantised by rows.
        dict(name="quantize_rows", op="quantize", rows=4099, cols=2048, dtype="bf16", scale="f32", form="rows"),
        # A training step's rows laid out along the tokens of each expert for the weights' gradient.
        dict(name="quantize_cols", op="quantize_cols", tokens=4096, topk=8, experts=32, parts=1, hidden=2048,
             dtype="bf16", scale="e8m0"),
        # One token through a dense 8-bit layer: bound by reading the weights once.
        dict(name="token_dense", op="matmul", rows=1, n=4096, k=7168, groups=0, scale="f32", out="bf16"),
        # One decode step of 64 tokens through 32 of 256 experts: one or two rows an expert.
        dict(name="decode_experts", op="matmul", tokens=64, topk=8, experts=256, parts=8, n=4096, k=7168, groups=32,
             scale="e8m0", out="bf16"),
        # A prefill of 8 ranks' 2048 tokens through 32 of 256 experts: the largest product.
        dict(name="prefill_experts", op="matmul", tokens=16384, topk=8, experts=256, parts=8, n=4096, k=7168,
             groups=32, scale="f32", out="bf16"),
        # The gradient of those experts' second weights, accumulated over the step's tokens in fp32.
        dict(name="wgrad_experts", op="wgrad", tokens=8192, topk=8, experts=256, parts=8, n=2048, k=7168, groups=32,
             scale="e8m0", out="f32"),
    ]


MOST_MACS = 16384 * 4096 * 7168  # of the largest listed product
MOST_WEIGHTS = 32 * 4096 * 7168
MOST_VALUES = 1 << 28            # of a drawn case's rows


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def _routing_sizes(rng, most_tokens):
    experts = rng.choice([8, 32, 64, 128, 160, 256])
    return dict(tokens=_log_uniform(rng, 1, most_tokens), topk=rng.choice([1, 2, 4, 6, 8]), experts=experts,
                parts=rng.choice([1, 1, 2, 8]))


def _width(rng):
    return rng.choice([1024, 2048, 2880, 4096, 5120, 7168, 8 * rng.randint(16, 1024), rng.randint(100, 8000)])


def draw(rng):
    op = rng.choice(["sort", "gather", "scatter", "scatter_grad", "quantize", "quantize_cols", "matmul", "matmul",
                     "experts", "experts", "wgrad"])
    scale = rng.choice(["f32", "e8m0"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "sort":
        return dict(op=op, **_routing_sizes(rng, 32768))
    if op == "quantize":
        cols = _width(rng)
        return dict(op=op, rows=_log_uniform(rng, 1, 16384), cols=cols, dtype=dtype, scale=scale,
                    form=rng.choice(["rows", "blocks"]))
    if op == "matmul":
        n, k = _width(rng), _width(rng)
        rows = _log_uniform(rng, 1, min(16384, MOST_MACS // (n * k)))
        return dict(op=op, rows=rows, n=n, k=k, groups=0, scale=scale, out=rng.choice(["bf16", "bf16", "f32"]))
    if op in ("experts", "wgrad"):
        c = _routing_sizes(rng, 16384)
        n, k = _width(rng), _width(rng)
        groups = c["experts"] // c["parts"]
        while groups * n * k > MOST_WEIGHTS // (4 if op == "wgrad" else 1):
            n, k = max(128, n // 2), max(128, k // 2)
        c["tokens"] = max(1, min(c["tokens"], MOST_MACS // 4 * c["parts"] // (c["topk"] * n * k)))
        return dict(op="matmul" if op == "experts" else op, **c, n=n, k=k, groups=groups, scale=scale,
                    out=rng.choice(["bf16", "bf16", "f32"]))
    hidden = _width(rng)
    c = _routing_sizes(rng, 16384)
    c["tokens"] = max(1, min(c["tokens"], MOST_VALUES // 4 * c["parts"] // (hidden * c["topk"])))
    c = dict(op=op, **c, hidden=hidden, dtype=dtype)
    if op == "gather":
        c["scale"] = rng.choice(["none", scale])
    elif op == "quantize_cols":
        c["scale"] = scale
    elif op == "scatter":
        c["weighted"] = rng.random() < 0.7
    return c


# ------------------------------------------------------------------ inputs

def _pad(n, m):
    return -(-n // m) * m


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _routing(case, gen):
    """int32 [T, k]: k distinct experts of each token; some experts are asked for more than others."""
    logits = torch.randn((case["tokens"], case["experts"]), generator=gen, device="cuda")
    logits += 0.3 * torch.randn((1, case["experts"]), generator=gen, device="cuda")
    return logits.topk(case["topk"], dim=1).indices.to(torch.int32).contiguous()


def _local(case):
    """(first expert, experts) of this rank: the last part but one."""
    count = case["experts"] // case["parts"]
    return count * max(0, case["parts"] - 2), count


def _capacity(case):
    """Rows that the program has room for, whatever the routing: every slot where all experts are here or the slots
    are few, otherwise twice what a part of many experts gets on average, and four times for a part of few."""
    count = case["experts"] // case["parts"]
    most = case["tokens"] * min(case["topk"], count)
    average = case["tokens"] * case["topk"] // case["parts"]
    return min(most, _pad((2 if count >= 16 else 4) * average + 64, 64))


def _rows(n, width, dtype, gen):
    """Activations: most channels near 1, a few much larger."""
    x = torch.randn((n, width), generator=gen, device="cuda")
    x *= torch.exp(torch.randn((1, width), generator=gen, device="cuda"))
    return x.to(DTYPES[dtype])


def _weights8(groups, n, k, scale, gen):
    w = torch.randn((groups, n, _pad(k, BLOCK)), generator=gen, device="cuda", dtype=torch.bfloat16)
    w[:, :, k:] = 0
    return _quantize_blocks(w, scale)


def _scale_buffer(scale, *shape):
    if scale == "f32":
        return torch.ones(shape, dtype=torch.float32, device="cuda")
    return torch.full(shape, 127, dtype=torch.uint8, device="cuda").view(E8M0)


def _pitch(k):
    """Scales in a row: the blocks of k values, to a multiple of four."""
    return _pad(_pad(k, BLOCK) // BLOCK, 4)


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    s = {"case": case}
    if "tokens" in case:
        s["topk"] = _routing(case, gen)
        s["first"], s["experts"] = _local(case)
        s["offsets"], s["slot_of"], s["row_of"] = _sort(s["topk"], s["first"], s["experts"])
        cap = s["cap"] = _capacity(case)
        s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
        T = case["tokens"]
    if op == "gather":
        s["x"] = _rows(T, case["hidden"], case["dtype"], gen)
        if case["scale"] == "none":
            s["out"] = torch.zeros((cap, case["hidden"]), dtype=DTYPES[case["dtype"]], device="cuda")
        else:
            s["out"] = torch.zeros((cap, _pad(case["hidden"], BLOCK)), dtype=torch.uint8, device="cuda").view(F8)
            s["scale"] = _scale_buffer(case["scale"], cap, _pitch(case["hidden"]))
    elif op == "scatter":
        s["y"] = _rows(cap, case["hidden"], case["dtype"], gen)
        s["weights"] = torch.rand((T, case["topk"]), generator=gen, device="cuda") if case["weighted"] else None
        s["out"] = torch.zeros((T, case["hidden"]), dtype=DTYPES[case["dtype"]], device="cuda")
    elif op == "scatter_grad":
        s["y"] = _rows(cap, case["hidden"], case["dtype"], gen)
        s["dout"] = _rows(T, case["hidden"], case["dtype"], gen)
        s["weights"] = torch.rand((T, case["topk"]), generator=gen, device="cuda")
        s["dy"] = torch.zeros((cap, case["hidden"]), dtype=DTYPES[case["dtype"]], device="cuda")
        s["dw"] = torch.zeros((T, case["topk"]), dtype=torch.float32, device="cuda")
    elif op == "quantize":
        rows, cols = case["rows"], case["cols"]
        s["x"] = _rows(rows, cols, case["dtype"], gen)
        s["out"] = torch.zeros((rows, _pad(cols, BLOCK)), dtype=torch.uint8, device="cuda").view(F8)
        srows = rows if case["form"] == "rows" else _pad(rows, BLOCK) // BLOCK
        s["scale"] = _scale_buffer(case["scale"], srows, _pitch(cols))
    elif op == "quantize_cols":
        s["x"] = _rows(T, case["hidden"], case["dtype"], gen)
        cols = _t_columns(cap, s["experts"])
        s["out"] = torch.zeros((case["hidden"], cols), dtype=torch.uint8, device="cuda").view(F8)
        s["scale"] = _scale_buffer(case["scale"], case["hidden"], _pitch(cols))
    elif op == "matmul":
        rows = case["rows"] if not case["groups"] else cap
        x = _rows(rows, case["k"], "bf16", gen)
        s["a"], s["a_scale"] = _quantize_rows(x, case["scale"])
        s["b"], s["b_scale"] = _weights8(max(1, case["groups"]), case["n"], case["k"], case["scale"], gen)
        s["out"] = torch.zeros((rows, case["n"]), dtype=DTYPES[case["out"]], device="cuda")
    elif op == "wgrad":
        for name, width in (("a", case["n"]), ("b", case["k"])):
            x = _rows(cap, width, "bf16", gen)
            s[name], s[name + "_scale"] = _quantize_cols(x, s["offsets"], case["scale"])
        s["out"] = torch.zeros((case["groups"], case["n"], case["k"]), dtype=DTYPES[case["out"]], device="cuda")
    return s


# ------------------------------------------------------------------ plain forms

def _sort(topk, first, experts):
    """Stable counting sort of the slots by expert, from a running count of each expert."""
    e = topk.reshape(-1).long() - first
    here = (e >= 0) & (e < experts)
    hot = e == torch.arange(experts, device=e.device).unsqueeze(1)
    upto = hot.cumsum(1, dtype=torch.int32)
    offsets = torch.zeros(experts + 1, dtype=torch.int32, device=e.device)
    offsets[1:] = upto[:, -1].cumsum(0)
    at = e.clamp(0, experts - 1)
    rank = upto.gather(0, at.unsqueeze(0)).squeeze(0) - 1
    row_of = torch.where(here, offsets[at] + rank, -1)
    slot_of = torch.full((e.numel() + 1,), -1, dtype=torch.int32, device=e.device)
    slots = torch.arange(e.numel(), dtype=torch.int32, device=e.device)
    slot_of[torch.where(here, row_of, e.numel()).long()] = torch.where(here, slots, -1)
    return offsets, slot_of[:-1], row_of.view(topk.shape)


def _scales(amax, scale):
    """(scale as it is kept, its value's reciprocal) of blocks whose largest magnitudes are amax."""
    s = amax / F8_MAX
    s = torch.where(s < SCALE_MIN, SCALE_MIN, s)
    s = torch.where(torch.isfinite(amax), s, math.nan)
    if scale == "f32":
        return s, 1.0 / s
    e = (s.view(torch.int32).long() + 0x7FFFFF) >> 23
    e = torch.where(torch.isnan(s), 255, e)
    r = torch.where(e == 255, math.nan, ((254 - e) << 23).to(torch.int32).view(torch.float32))
    return e.to(torch.uint8).view(E8M0), r


def _scale_value(scale):
    """fp32 values of kept scales."""
    return scale if scale.dtype == torch.float32 else torch.exp2(scale.view(torch.uint8).float() - 127)


def _padded(x, dim, n, value=0):
    if x.shape[dim] == n:
        return x
    shape = list(x.shape)
    shape[dim] = n
    out = torch.full(shape, value, dtype=x.dtype, device=x.device)
    out.narrow(dim, 0, x.shape[dim]).copy_(x)
    return out


def _padded_scale(s, pitch):
    """Scales in rows of `pitch`, ones past the last block."""
    if s.dtype == torch.float32:
        return _padded(s, -1 % s.dim(), pitch, 1.0)
    return _padded(s.view(torch.uint8), -1 % s.dim(), pitch, 127).view(E8M0)


def _quantize_rows(x, scale):
    rows, k = x.shape
    v = _padded(x.float(), 1, _pad(k, BLOCK)).view(rows, -1, BLOCK)
    kept, r = _scales(v.abs().amax(2), scale)
    return (v * r.unsqueeze(2)).to(F8).view(rows, -1), _padded_scale(kept, _pitch(k))


def _quantize_blocks(w, scale):
    """w [.., n, k] in blocks of 128 x 128."""
    n, k = w.shape[-2:]
    kp, np_ = _pad(k, BLOCK), _pad(n, BLOCK)
    v = _padded(_padded(w.reshape(-1, n, k), 2, kp), 1, np_).float().view(-1, np_ // BLOCK, BLOCK, kp // BLOCK, BLOCK)
    kept, r = _scales(v.abs().amax((2, 4)), scale)
    q = (v * r[:, :, None, :, None]).to(F8).view(-1, np_, kp)[:, :n].contiguous()
    return q.view(*w.shape[:-1], kp), _padded_scale(kept, _pitch(k)).view(*w.shape[:-2], np_ // BLOCK, -1)


def _t_columns(rows, groups):
    """Columns of rows laid out along the tokens: every group starts at a block of 128 of its own."""
    return BLOCK * (rows // BLOCK + groups)


def _t_places(offsets, rows):
    """(column of each row, whether the row belongs to a group) of that layout: group g starts at block
    offsets[g] / 128 + g."""
    r = torch.arange(rows, device=offsets.device)
    off = offsets.long()
    g = (r.unsqueeze(1) >= off[1:]).sum(1)
    used = g < off.numel() - 1
    g = g.clamp(max=off.numel() - 2)
    return (off[g] // BLOCK + g) * BLOCK + r - off[g], used


def _quantize_cols(x, offsets, scale):
    """x [rows, H] -> [H, columns] with a scale per 128 rows of a group."""
    rows, width = x.shape
    cols = _t_columns(rows, offsets.numel() - 1)
    place, used = _t_places(offsets, rows)
    v = torch.zeros((cols, width), dtype=torch.float32, device=x.device)
    v[place[used]] = x[used].float()
    v = v.view(-1, BLOCK, width)
    kept, r = _scales(v.abs().amax(1), scale)
    q = (v * r.unsqueeze(1)).to(F8).view(cols, width)
    kept = kept.view(torch.uint8).t().contiguous().view(E8M0) if scale == "e8m0" else kept.t().contiguous()
    return q.view(torch.uint8).t().contiguous().view(F8), _padded_scale(kept, _pitch(cols))


def _dequantized(q, scale, row_block=1):
    """fp32 values of q [.., n, k] with a scale per 128 columns of every `row_block` rows."""
    v = q.float()
    n, k = v.shape[-2:]
    s = _scale_value(scale)[..., :k // BLOCK]
    if row_block > 1:
        s = s.repeat_interleave(row_block, dim=-2)[..., :n, :]
    return (v.view(*v.shape[:-1], k // BLOCK, BLOCK) * s.unsqueeze(-1)).view(v.shape)


def _group_rows(s):
    """int64 [groups, most]: the rows of each group, the last row's successor (a row of zeros) past its end."""
    off = s["offsets"].long()
    r = off[:-1].unsqueeze(1) + torch.arange(max(1, s["most"]), device=off.device)
    return torch.where(r < off[1:].unsqueeze(1), r, s["cap"])


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "sort":
        return _sort(s["topk"], s["first"], s["experts"])
    if op == "quantize":
        return (_quantize_rows if case["form"] == "rows" else _quantize_blocks)(s["x"], case["scale"])
    if op == "matmul" and not case["groups"]:
        a = _dequantized(s["a"], s["a_scale"])
        b = _dequantized(s["b"], s["b_scale"], BLOCK)[0]
        return (a @ b.t()).to(s["out"].dtype)
    if op == "matmul":
        rows = _group_rows(s)
        a = _padded(_dequantized(s["a"], s["a_scale"]), 0, s["cap"] + 1)[rows]
        c = torch.bmm(a, _dequantized(s["b"], s["b_scale"], BLOCK).transpose(1, 2))
        out = torch.zeros((s["cap"] + 1, case["n"]), dtype=torch.float32, device=a.device)
        out[rows] = c
        return out[:-1].to(s["out"].dtype)
    if op == "wgrad":
        place, used = _t_places(s["offsets"], s["cap"])
        rows = _group_rows(s)
        a, b = (_padded(_dequantized(s[m], s[m + "_scale"]).t()[place] * used.unsqueeze(1), 0, s["cap"] + 1)[rows]
                for m in ("a", "b"))
        return torch.bmm(a.transpose(1, 2), b).to(s["out"].dtype)
    row_of = s["row_of"].long()
    here = row_of >= 0
    if op == "gather":
        token = torch.arange(case["tokens"], device=row_of.device).unsqueeze(1).expand_as(row_of)[here]
        if case["scale"] == "none":
            out = torch.zeros_like(s["out"])
            out[row_of[here]] = s["x"][token]
            return out
        x = torch.zeros((s["cap"], case["hidden"]), dtype=torch.float32, device=row_of.device)
        x[row_of[here]] = s["x"][token].float()
        q, scale = _quantize_rows(x, case["scale"])
        unused = torch.arange(s["cap"], device=row_of.device) >= s["offsets"][-1]
        kept = torch.where(unused.unsqueeze(1), 127 if case["scale"] == "e8m0" else 1.0,
                           scale.view(torch.uint8) if case["scale"] == "e8m0" else scale)
        return q, kept.to(torch.uint8).view(E8M0) if case["scale"] == "e8m0" else kept
    if op == "quantize_cols":
        slot = s["slot_of"][:s["cap"]].long()
        x = s["x"][slot.clamp(min=0) // case["topk"]]
        return _quantize_cols(x, s["offsets"], case["scale"])
    y = s["y"].float()[row_of.clamp(min=0)]  # [T, k, H]
    w = torch.ones(row_of.shape, device=y.device) if s["weights"] is None else s["weights"]
    if op == "scatter":
        terms = torch.where(here.unsqueeze(2), w.unsqueeze(2) * y, 0.0)
        return terms.sum(1).to(s["out"].dtype)
    dout = s["dout"].float()
    dw = torch.where(here, (y * dout.unsqueeze(1)).sum(2), 0.0)
    dy = torch.zeros((s["cap"], case["hidden"]), dtype=torch.float32, device=y.device)
    dy[row_of[here]] = (w.unsqueeze(2) * dout.unsqueeze(1))[here]
    return dy.to(s["dy"].dtype), dw


def _own(s):
    from paper_2608_00867_amd import nuna
    case = s["case"]
    op = case["op"]
    if op == "sort":
        return nuna.moe_sort(s["topk"], s["experts"], s["first"])
    if op == "gather":
        if case["scale"] == "none":
            return nuna.moe_gather(s["x"], s["row_of"], s["out"])
        return nuna.moe_gather(s["x"], s["row_of"], s["out"], s["scale"])
    if op == "scatter":
        return nuna.moe_scatter(s["y"], s["row_of"], s["weights"], s["out"])
    if op == "scatter_grad":
        return nuna.moe_scatter_grad(s["dout"], s["y"], s["row_of"], s["weights"], s["dy"], s["dw"])
    if op == "quantize":
        quantize = nuna.f8_quantize if case["form"] == "rows" else nuna.f8_quantize_blocks
        return quantize(s["x"], case["scale"], s["out"], s["scale"])
    if op == "quantize_cols":
        return nuna.f8_quantize_cols(s["x"], s["offsets"], case["scale"], s["out"], s["scale"],
                                     slot_of=s["slot_of"][:s["cap"]], topk=case["topk"])
    if op == "matmul":
        return nuna.f8_matmul(s["a"], s["a_scale"], s["b"] if case["groups"] else s["b"][0],
                              s["b_scale"] if case["groups"] else s["b_scale"][0], s["out"],
                              offsets=s["offsets"] if case["groups"] else None)
    return nuna.f8_wgrad(s["a"], s["a_scale"], s["b"], s["b_scale"], s["offsets"], s["out"])


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ work

def _scale_bytes(rows, k, scale):
    return rows * _pad(k, BLOCK) // BLOCK * (4 if scale == "f32" else 1)


def work(case):
    op = case["op"]
    if op == "quantize":
        values = case["rows"] * case["cols"]
        srows = case["rows"] if case["form"] == "rows" else _pad(case["rows"], BLOCK) // BLOCK
        return {"bytes": values * (ESIZE[case["dtype"]] + 1) + _scale_bytes(srows, case["cols"], case["scale"]),
                "flops": 2 * values}
    if op == "matmul" and not case["groups"]:
        rows, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": (rows + n) * k + rows * n * ESIZE[case["out"]] + _scale_bytes(rows, k, case["scale"]) +
                _scale_bytes(_pad(n, BLOCK) // BLOCK, k, case["scale"]), "flops": 2 * rows * n * k}
    T, k, E, count = case["tokens"], case["topk"], case["experts"], case["experts"] // case["parts"]
    slots = T * k
    if op == "sort":
        return {"bytes": 12 * slots + 4 * (count + 1), "flops": 0}
    rows = slots / case["parts"]
    reached = T * (1 - math.comb(E - count, k) / math.comb(E, k))  # tokens that have an expert here
    if op in ("matmul", "wgrad"):
        n, w = case["n"], case["k"]
        live = count * (1 - (1 - 1 / E) ** slots)  # experts that have a row
        flops = 2 * rows * n * w
        if op == "matmul":
            return {"bytes": live * n * w + rows * (w + n * ESIZE[case["out"]]), "flops": flops}
        return {"bytes": rows * (n + w) + count * n * w * ESIZE[case["out"]], "flops": flops}
    H, es = case["hidden"], ESIZE[case["dtype"]]
    if op == "gather":
        to = es * H if case["scale"] == "none" else H + _scale_bytes(1, H, case["scale"])
        return {"bytes": reached * H * es + rows * to + 4 * slots, "flops": 0 if case["scale"] == "none" else 2 * reached * H}
    if op == "quantize_cols":
        return {"bytes": reached * H * es + rows * H + _scale_bytes(H, rows, case["scale"]), "flops": 2 * rows * H}
    if op == "scatter":
        return {"bytes": (rows + T) * H * es + 4 * slots * (2 if case["weighted"] else 1),
                "flops": (2 if case["weighted"] else 1) * rows * H}
    return {"bytes": (2 * rows + reached) * H * es + 12 * slots, "flops": 3 * rows * H}


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_e4m3(v):
    """Float64 values rounded to the nearest e4m3 value, ties to even: 3 bits of fraction from 2^-6 up, steps of 2^-9
    below."""
    e = torch.frexp(v.abs().clamp(min=2.0 ** -20))[1] - 1
    step = torch.exp2(e.clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def _exact_scale(amax, scale):
    s = (amax / F8_MAX).clamp(min=SCALE_MIN)
    return s if scale == "f32" else torch.exp2(torch.ceil(torch.log2(s)))


def _exact_kept(s, pitch):
    """Scales in rows of `pitch` as float64, ones past the last block."""
    out = torch.ones((*s.shape[:-1], pitch), dtype=torch.float64, device=s.device)
    out[..., :s.shape[-1]] = s
    return out


def _exact_quantized(x, scale, along_rows):
    """x float64 [n, k], k whole blocks: (q values, scales [n or n / 128, k / 128])."""
    n, k = x.shape
    v = x.view(n, k // BLOCK, BLOCK)
    amax = v.abs().amax(2)
    if not along_rows:
        amax = torch.stack([amax[i:i + BLOCK].amax(0) for i in range(0, n, BLOCK)])
    s = _exact_scale(amax, scale)
    per_row = s if along_rows else s.repeat_interleave(BLOCK, 0)[:n]
    return _exact_e4m3(v / per_row.unsqueeze(2)).view(n, k), s


def _widened(x):
    out = torch.zeros((x.shape[0], _pad(x.shape[1], BLOCK)), dtype=torch.float64, device=x.device)
    out[:, :x.shape[1]] = x
    return out


def _exact_values(q, scale):
    """Float64 values of a stored matrix [n, k] with a scale per row and block."""
    blocks = q.shape[1] // BLOCK
    s = scale.double() if scale.dtype == torch.float32 else torch.exp2(scale.view(torch.uint8).double() - 127)
    return q.float().double() * s[:, :blocks].repeat_interleave(BLOCK, 1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        q, sc = _exact_quantized(_widened(s["x"].double()), case["scale"], case["form"] == "rows")
        return q, _exact_kept(sc, _pitch(case["cols"]))
    if op == "matmul" and not case["groups"]:
        b = _exact_values(s["b"][0], s["b_scale"][0].view(torch.uint8 if case["scale"] == "e8m0" else torch.float32)
                          .repeat_interleave(BLOCK, 0)[:case["n"]])
        return _exact_values(s["a"], s["a_scale"]) @ b.t()
    off = s["offsets"].tolist()
    if op == "matmul":
        out = torch.zeros((s["cap"], case["n"]), dtype=torch.float64, device="cuda")
        a = _exact_values(s["a"], s["a_scale"])
        for g in range(case["groups"]):
            if off[g] < off[g + 1]:
                sb = s["b_scale"][g].view(torch.uint8 if case["scale"] == "e8m0" else torch.float32)
                b = _exact_values(s["b"][g], sb.repeat_interleave(BLOCK, 0)[:case["n"]])
                out[off[g]:off[g + 1]] = a[off[g]:off[g + 1]] @ b.t()
        return out
    if op == "wgrad":
        out = torch.zeros((case["groups"], case["n"], case["k"]), dtype=torch.float64, device="cuda")
        a, b = (_exact_values(s[m], s[m + "_scale"]) for m in ("a", "b"))
        for g in range(case["groups"]):
            at, rows = BLOCK * (off[g] // BLOCK + g), off[g + 1] - off[g]
            out[g] = a[:, at:at + rows] @ b[:, at:at + rows].t().contiguous()
        return out
    e = s["topk"].reshape(-1).long()
    if op == "sort":
        local = torch.where((e >= s["first"]) & (e < s["first"] + s["experts"]), e, 1 << 30)
        order = torch.sort(local, stable=True).indices
        used = off[-1]
        slot_of = torch.where(torch.arange(e.numel(), device="cuda") < used, order, -1)
        row_of = torch.full_like(e, -1)
        row_of[order[:used]] = torch.arange(used, device="cuda")
        counts = torch.stack([(local < s["first"] + g).sum() for g in range(s["experts"] + 1)])
        return counts, slot_of, row_of.view(s["topk"].shape)
    slot = s["slot_of"].long()[:off[-1]]
    token = slot // case["topk"]
    H = case["hidden"]
    if op == "gather":
        x = s["x"].double()
        if case["scale"] == "none":
            out = torch.zeros((s["cap"], H), dtype=torch.float64, device="cuda")
            out[:off[-1]] = x[token]
            return out
        q, sc = _exact_quantized(_widened(x), case["scale"], True)
        out = torch.zeros((s["cap"], q.shape[1]), dtype=torch.float64, device="cuda")
        out[:off[-1]] = q[token]
        kept = torch.ones((s["cap"], _pitch(H)), dtype=torch.float64, device="cuda")
        kept[:off[-1]] = _exact_kept(sc, _pitch(H))[token]
        return out, kept
    if op == "quantize_cols":
        cols = _t_columns(s["cap"], s["experts"])
        v = torch.zeros((cols, H), dtype=torch.float64, device="cuda")
        for g in range(s["experts"]):
            at = BLOCK * (off[g] // BLOCK + g)
            v[at:at + off[g + 1] - off[g]] = s["x"].double()[token[off[g]:off[g + 1]]]
        q, sc = _exact_quantized(v.t().contiguous(), case["scale"], True)
        return q, _exact_kept(sc, _pitch(cols))
    y = torch.zeros((s["topk"].numel(), H), dtype=torch.float64, device="cuda")
    y[slot] = s["y"][:off[-1]].double()
    y = y.view(case["tokens"], case["topk"], H)
    if op == "scatter":
        return (y if s["weights"] is None else y * s["weights"].double().unsqueeze(2)).sum(1)
    dout = s["dout"].double()
    dy = torch.zeros((s["cap"], H), dtype=torch.float64, device="cuda")
    dy[:off[-1]] = dout[token] * s["weights"].double().view(-1)[slot].unsqueeze(1)
    return dy, (y * dout.unsqueeze(1)).sum(2)
