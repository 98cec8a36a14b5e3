"""Cases of what stands around the expert layer's operators in a transformer block: the root-mean-square norm with the
residual's addition, the router that writes the top-k tables, SwiGLU between the experts' two products, and a whole expert
layer for a few tokens.

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
EPS = 1e-6
FACTOR = 2.5  # of the router's weights where they are normalised


def listed():
    return [
        # One decode step of 64 sequences: residual added, normed and quantised for the next 8-bit product.
        dict(name="norm_decode", op="norm", tokens=64, hidden=7168, dtype="bf16", residual=True, scale="e8m0"),
        # A training step's norm (an odd number of tokens), the statistics kept for the backward pass.
        dict(name="norm_train", op="norm", tokens=8195, hidden=2880, dtype="bf16", residual=True, scale="none"),
        # The backward pass of the same kind of step at a wide model; the residual's own gradient comes in.
        dict(name="norm_grad", op="norm_grad", tokens=4096, hidden=7168, dtype="bf16", residual=True),
        # Router of one decode step: sigmoid scores, chosen with a balancing bias, fp32 logits.
        dict(name="route_decode", op="route", tokens=64, topk=8, experts=256, dtype="f32", score="sigmoid", bias=True,
             normalize=True, masked=False),
        # Router of a long prefill, an odd number of tokens; softmax over bf16 logits, padded rows and an expert that is
        # out of service.
        dict(name="route_prefill", op="route", tokens=32771, topk=8, experts=256, dtype="bf16", score="softmax",
             bias=False, normalize=True, masked=True),
        # The router's backward pass, softmax over all experts.
        dict(name="route_grad", op="route_grad", tokens=16384, topk=4, experts=32, dtype="f32", score="softmax",
             normalize=False, masked=False),
        # Between the experts' products of a prefill on one of 8 ranks: fp32 scales for the second product.
        dict(name="swiglu_prefill", op="swiglu", tokens=16384, topk=8, experts=256, parts=8, inner=2048, dtype="bf16",
             scale="f32", also=False),
        # The same in a training step, which keeps the 16-bit result too; a width that is no multiple of 128.
        dict(name="swiglu_train", op="swiglu", tokens=4099, topk=4, experts=32, parts=1, inner=2888, dtype="bf16",
             scale="e8m0", also=True),
        # Its backward pass: the gradient in 16 bits for the weights' gradient, in 8 for the rows' product.
        dict(name="swiglu_grad", op="swiglu_grad", tokens=4096, topk=8, experts=256, parts=8, inner=2048, dtype="bf16",
             scale="e8m0", also=True),
        # One token through its 8 of 32 experts: bound by reading their weights once.
        dict(name="few_token", op="few", tokens=1, topk=8, experts=32, parts=1, hidden=7168, inner=2048, dtype="bf16",
             scale="e8m0"),
        # A decode step of 64 tokens on one of 8 ranks of 256 experts: nearly all 32 are reached, by one or two tokens.
        dict(name="few_batch", op="few", tokens=64, topk=8, experts=256, parts=8, hidden=7168, inner=2048,
             dtype="bf16", scale="f32"),
        # A few sequences of a small model in fp32, widths that are no multiple of 128.
        dict(name="few_f32", op="few", tokens=7, topk=4, experts=32, parts=1, hidden=2880, inner=1440, dtype="f32",
             scale="f32"),
    ]


MOST_VALUES = 4096 * 7168 * 3        # of a drawn case's widest matrix
MOST_WEIGHTS = 32 * 3 * 7168 * 2048  # of the largest listed layer


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def _routing_sizes(rng, most_tokens):
    experts = rng.choice([8, 32, 64, 128, 160, 256])
    return dict(tokens=_log_uniform(rng, 1, most_tokens), topk=rng.choice([1, 2, 4, 6, 8]), experts=experts,
                parts=rng.choice([1, 1, 2, 8]))


def _width(rng, most=8192):
    return min(most, rng.choice([512, 1024, 2048, 2880, 4096, 5120, 7168, 8192, 8 * rng.randint(16, 1024),
                                 rng.randint(100, 8000)]))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "route", "route", "route_grad", "swiglu", "swiglu_grad", "few", "few",
                     "few"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    scale = rng.choice(["f32", "e8m0"])
    if op in ("norm", "norm_grad"):
        hidden = _width(rng)
        c = dict(op=op, tokens=_log_uniform(rng, 1, min(32768, MOST_VALUES // (3 * hidden * (ESIZE[dtype] // 2)))),
                 hidden=hidden, dtype=dtype, residual=rng.random() < 0.7)
        if op == "norm":
            c["scale"] = rng.choice(["none", scale])
        return c
    if op in ("route", "route_grad"):
        experts = rng.choice([8, 32, 64, 100, 128, 160, 256, 512])
        c = dict(op=op, tokens=_log_uniform(rng, 1, 32768 * 256 // max(256, experts)),
                 topk=rng.choice([k for k in (1, 2, 4, 6, 8, 10) if k <= experts]), experts=experts,
                 dtype=rng.choice(["bf16", "f32"]), score=rng.choice(["softmax", "sigmoid"]),
                 normalize=rng.random() < 0.7, masked=rng.random() < 0.4)
        if op == "route":
            c["bias"] = c["score"] == "sigmoid" and rng.random() < 0.7
        return c
    c = _routing_sizes(rng, 64 if op == "few" else 16384)
    if op == "few":
        hidden, inner = _width(rng, 7168), _width(rng, 4096)
        while c["experts"] // c["parts"] * 3 * hidden * inner > MOST_WEIGHTS:
            hidden, inner = max(256, hidden // 2), max(128, inner // 2)
        return dict(op=op, **c, hidden=hidden, inner=inner, dtype=dtype, scale=scale)
    inner = _width(rng)
    most = MOST_VALUES // (3 * inner * (ESIZE[dtype] // 2))
    c["tokens"] = max(1, min(c["tokens"], most * c["parts"] // (2 * c["topk"])))
    scale = rng.choice(["none", scale, scale])
    return dict(op=op, **c, inner=inner, dtype=dtype, scale=scale, also=scale != "none" and rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

def _pad(n, m):
    return -(-n // m) * m


def _pitch(k):
    """Scales in a row: the blocks of k values, to a multiple of four."""
    return _pad(_pad(k, BLOCK) // BLOCK, 4)


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _logits(case, gen, spread=1.5):
    """fp32 [T, E] router logits; some experts are asked for more than others."""
    z = spread * torch.randn((case["tokens"], case["experts"]), generator=gen, device="cuda")
    return z + 0.3 * torch.randn((1, case["experts"]), generator=gen, device="cuda")


def _local(case):
    """(first expert, experts) of this rank: the last part but one."""
    count = case["experts"] // case["parts"]
    return count * max(0, case["parts"] - 2), count


def _rows(n, width, dtype, gen):
    """Activations: most channels near 1, a few much larger."""
    x = torch.randn((n, width), generator=gen, device="cuda")
    x *= torch.exp(torch.randn((1, width), generator=gen, device="cuda"))
    return x.to(DTYPES[dtype])


def _weights8(groups, n, k, scale, gen):
    """Weights [groups, n, k] near 1 / sqrt(k), in 8 bits with a scale for each block of 128 x 128."""
    kp, np_ = _pad(k, BLOCK), _pad(n, BLOCK)
    w = torch.randn((groups, np_, kp), generator=gen, device="cuda", dtype=torch.bfloat16) * k ** -0.5
    w[:, n:] = 0
    w[:, :, k:] = 0
    v = w.view(groups, np_ // BLOCK, BLOCK, kp // BLOCK, BLOCK)
    kept, r = _scales(v.abs().amax((2, 4)).float(), scale)
    q = (v * r[:, :, None, :, None].bfloat16()).to(F8) if scale == "e8m0" else (v * r[:, :, None, :, None]).to(F8)
    return q.view(groups, np_, kp)[:, :n].contiguous(), _padded_scale(kept, _pitch(k))


def _f8_buffers(s, rows, cols, scale):
    s["q"] = torch.zeros((rows, _pad(cols, BLOCK)), dtype=torch.uint8, device="cuda").view(F8)
    if scale == "f32":
        s["q_scale"] = torch.ones((rows, _pitch(cols)), dtype=torch.float32, device="cuda")
    else:
        s["q_scale"] = torch.full((rows, _pitch(cols)), 127, dtype=torch.uint8, device="cuda").view(E8M0)


def prepare(case, seed):
    gen = _generator(seed)
    op = case["op"]
    s = {"case": case}
    T = case["tokens"]
    dt = DTYPES[case["dtype"]]
    if op in ("norm", "norm_grad"):
        H = case["hidden"]
        s["x"] = _rows(T, H, case["dtype"], gen)
        s["weight"] = (1 + 0.2 * torch.randn(H, generator=gen, device="cuda")).to(dt)
        if case["residual"]:
            s["residual"] = _rows(T, H, case["dtype"], gen)
        if op == "norm":
            s["z"] = torch.zeros((T, H), dtype=dt, device="cuda")
            if case["scale"] == "none":
                s["out"] = torch.zeros((T, H), dtype=dt, device="cuda")
                s["rstd"] = torch.zeros(T, dtype=torch.float32, device="cuda")
            else:
                _f8_buffers(s, T, H, case["scale"])
        else:
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + EPS)
            s["dout"] = _rows(T, H, case["dtype"], gen)
            s["dx"] = torch.zeros((T, H), dtype=dt, device="cuda")
        return s
    if op in ("route", "route_grad"):
        z = _logits(case, gen)
        if case["masked"]:
            z[:, torch.randint(case["experts"], (1,), generator=gen, device="cuda")] = -math.inf
            z[torch.rand(T, generator=gen, device="cuda") < 0.05] = -math.inf
        s["logits"] = z.to(dt)
        s["bias"] = 0.1 * torch.randn(case["experts"], generator=gen, device="cuda") if case.get("bias") else None
        if op == "route_grad":
            s["topk_idx"] = _chosen(s["logits"], None, case)
            s["dweights"] = torch.randn((T, case["topk"]), generator=gen, device="cuda")
        return s
    s["topk_idx"] = _logits(case, gen, 1.0).topk(case["topk"], dim=1).indices.to(torch.int32).contiguous()
    s["first"], s["experts"] = _local(case)
    if op == "few":
        H, inner = case["hidden"], case["inner"]
        s["x"] = _rows(T, H, case["dtype"], gen)
        w = torch.rand((T, case["topk"]), generator=gen, device="cuda") + 0.1
        s["weights"] = w / w.sum(1, keepdim=True)
        s["w1"], s["w1_scale"] = _weights8(s["experts"], 2 * inner, H, case["scale"], gen)
        s["w2"], s["w2_scale"] = _weights8(s["experts"], H, inner, case["scale"], gen)
        s["out"] = torch.zeros((T, H), dtype=dt, device="cuda")
        return s
    # Rows in expert order: as many as the routing brings here, in a buffer that has room for more.
    local = s["topk_idx"].long() - s["first"]
    counts = torch.zeros(s["experts"] + 1, dtype=torch.int64, device="cuda")
    counts.index_add_(0, torch.where((local >= 0) & (local < s["experts"]), local + 1, 0).view(-1),
                      ((local >= 0) & (local < s["experts"])).long().view(-1))
    s["offsets"] = counts.cumsum(0).to(torch.int32)
    most = T * min(case["topk"], s["experts"])
    cap = s["cap"] = min(most, _pad(2 * T * case["topk"] // case["parts"] + 64, 64))
    inner = case["inner"]
    s["gu"] = _rows(cap, 2 * inner, case["dtype"], gen)
    wide = inner
    if op == "swiglu_grad":
        s["dout"] = _rows(cap, inner, case["dtype"], gen)
        wide = 2 * inner
    if case["scale"] != "none":
        _f8_buffers(s, cap, wide, case["scale"])
    if case["scale"] == "none" or case["also"]:
        s["out"] = torch.zeros((cap, wide), dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms

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


def _dequantized(q, scale):
    """fp32 values of q [.., n, k] with a scale per block of 128 x 128."""
    n, k = q.shape[-2:]
    s = scale if scale.dtype == torch.float32 else torch.exp2(scale.view(torch.uint8).float() - 127)
    s = s[..., :k // BLOCK].repeat_interleave(BLOCK, dim=-2)[..., :n, :]
    return (q.float().view(*q.shape[:-1], k // BLOCK, BLOCK) * s.unsqueeze(-1)).view(q.shape)


def _alive(z, bias):
    """Experts that can be chosen: those whose logit (and bias) is above -inf."""
    alive = z > -math.inf
    return alive if bias is None else alive & (bias > -math.inf)


def _chosen(logits, bias, case):
    """int32 [T, k]: the experts of the largest scores, the lowest first among equals; -1 where none is left.  The
    scores of the biased choice lie close together, so they are formed in 64 bits."""
    z = logits.double()
    key = z if bias is None else 1 / (1 + torch.exp(-z)) + bias.double()
    alive = _alive(z, bias)
    order = torch.sort(torch.where(alive, key, -math.inf), dim=1, descending=True, stable=True).indices[:, :case["topk"]]
    return torch.where(alive.gather(1, order), order, -1).to(torch.int32).contiguous()


def _scores(logits, score):
    """Scores of all experts before they are normalised: softmax's exponentials relative to the row's largest, or
    sigmoids."""
    z = logits.float()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    top = z.amax(1, keepdim=True)
    return torch.exp(z - torch.where(top > -math.inf, top, 0.0))


def _gate(p, idx, score, normalize):
    """(chosen scores [T, k], the sums that they are divided by [T, 1])."""
    here = idx >= 0
    chosen = torch.where(here, p.gather(1, idx.long().clamp(min=0)), 0.0)
    total = chosen.sum(1, keepdim=True) if normalize else \
        p.sum(1, keepdim=True) if score == "softmax" else torch.ones_like(chosen[:, :1])
    return chosen, torch.where(total > 0, total, 1.0)


def _factor(case):
    return FACTOR if case["normalize"] else 1.0


def _used(s):
    """[rows, 1]: rows that belong to an expert."""
    return (torch.arange(s["cap"], device="cuda") < s["offsets"][-1]).unsqueeze(1)


def _quantized_used(v, used, scale):
    q, kept = _quantize_rows(v, scale)
    if scale == "e8m0":
        return q, torch.where(used, kept.view(torch.uint8), 127).view(E8M0)
    return q, torch.where(used, kept, 1.0)


def _plain(s):
    case = s["case"]
    op = case["op"]
    dt = DTYPES[case["dtype"]]
    if op == "norm":
        z = s["x"]
        if case["residual"]:
            z = (z.float() + s["residual"].float()).to(dt)
        v = z.float()
        rstd = 1 / torch.sqrt((v * v).sum(1, keepdim=True) / case["hidden"] + EPS)
        y = v * rstd * s["weight"].float()
        first = (z,) if case["residual"] else ()
        if case["scale"] == "none":
            return (*first, y.to(dt), rstd.squeeze(1))
        return (*first, *_quantize_rows(y, case["scale"]))
    if op == "norm_grad":
        v, g, r = s["x"].float(), s["dout"].float(), s["rstd"].unsqueeze(1)
        zhat = v * r
        u = g * s["weight"].float()
        dx = r * (u - zhat * ((u * zhat).sum(1, keepdim=True) / case["hidden"]))
        if case["residual"]:
            dx = dx + s["residual"].float()
        return dx.to(dt), (g * zhat).sum(0)
    if op == "route":
        idx = _chosen(s["logits"], s["bias"], case)
        chosen, total = _gate(_scores(s["logits"], case["score"]), idx, case["score"], case["normalize"])
        return idx, _factor(case) * chosen / total
    if op == "route_grad":
        idx, g, f = s["topk_idx"], s["dweights"], _factor(case)
        p = _scores(s["logits"], case["score"])
        chosen, total = _gate(p, idx, case["score"], case["normalize"])
        q = chosen / total
        at = torch.where(idx >= 0, idx.long(), case["experts"])
        dz = torch.zeros((case["tokens"], case["experts"] + 1), dtype=torch.float32, device="cuda")
        if case["normalize"]:
            each = f * q * (g - (q * g).sum(1, keepdim=True))
            if case["score"] == "sigmoid":
                each = each * (1 - chosen)
            dz = dz.scatter_add(1, at, each)[:, :-1]
        elif case["score"] == "sigmoid":
            dz = dz.scatter_add(1, at, f * g * q * (1 - q))[:, :-1]
        else:
            dz = f * (p / total) * (dz.scatter_add(1, at, g)[:, :-1] - (q * g).sum(1, keepdim=True))
        return dz.to(dt)
    if op == "few":
        local = s["topk_idx"].long() - s["first"]
        here = (local >= 0) & (local < s["experts"])
        T, k = local.shape
        if T * k < s["experts"]:  # a layer for each slot
            e = local.clamp(0, s["experts"] - 1).view(-1)
            w1 = _dequantized(s["w1"].view(torch.uint8)[e].view(F8), _scale_rows(s["w1_scale"], e))
            w2 = _dequantized(s["w2"].view(torch.uint8)[e].view(F8), _scale_rows(s["w2_scale"], e))
            x = s["x"].float().unsqueeze(1).expand(T, k, -1).reshape(T * k, 1, -1)
            y = _swiglu_layer(x, w1, w2, case).view(T, k, -1)
            return torch.where(here.unsqueeze(2), s["weights"].unsqueeze(2) * y, 0.0).sum(1).to(dt)
        w1, w2 = _dequantized(s["w1"], s["w1_scale"]), _dequantized(s["w2"], s["w2_scale"])
        y = _swiglu_layer(s["x"].float().unsqueeze(0), w1, w2, case)  # [E, T, H]
        hot = local.unsqueeze(0) == torch.arange(s["experts"], device="cuda").view(-1, 1, 1)
        w = torch.where(hot, s["weights"], 0.0).sum(2, keepdim=True)  # [E, T, 1]
        return torch.where(hot.any(2, keepdim=True), w * y, 0.0).sum(0).to(dt)
    used = _used(s)
    gate, up = s["gu"][:, :case["inner"]].float(), s["gu"][:, case["inner"]:].float()
    sig = 1 / (1 + torch.exp(-gate))
    if op == "swiglu":
        v = gate * sig * up
    else:
        g = s["dout"].float()
        v = torch.cat([g * up * (sig * (1 + gate * (1 - sig))), g * gate * sig], 1)
    v = torch.where(used, v, 0.0)
    full = (v.to(dt),) if "out" in s else ()
    return full if case["scale"] == "none" else (*full, *_quantized_used(v, used, case["scale"]))


def _scale_rows(scale, e):
    return scale[e] if scale.dtype == torch.float32 else scale.view(torch.uint8)[e].view(E8M0)


def _swiglu_layer(x, w1, w2, case):
    """x [.., T, H] through w1 [B, 2 I, H padded] and w2 [B, H, I padded], in fp32."""
    H, inner = case["hidden"], case["inner"]
    gu = torch.matmul(x, w1[:, :, :H].transpose(1, 2))
    gate, up = gu[..., :inner], gu[..., inner:]
    h = gate / (1 + torch.exp(-gate)) * up
    return torch.matmul(h, w2[:, :, :inner].transpose(1, 2))


def _own(s):
    from paper_2608_00867_amd import nuna
    case = s["case"]
    op = case["op"]
    if op == "norm":
        first = (s["z"],) if case["residual"] else ()
        residual = dict(residual=s["residual"], residual_out=s["z"]) if case["residual"] else {}
        if case["scale"] == "none":
            out = nuna.rms_norm(s["x"], s["weight"], EPS, out=s["out"], rstd=s["rstd"], **residual)
            return (*first, out, s["rstd"])
        return (*first, *nuna.rms_norm(s["x"], s["weight"], EPS, scale=case["scale"], q_out=s["q"],
                                       scale_out=s["q_scale"], **residual))
    if op == "norm_grad":
        return nuna.rms_norm_grad(s["dout"], s["x"], s["weight"], s["rstd"], dresidual=s.get("residual"), dx=s["dx"])
    if op == "route":
        return nuna.route_topk(s["logits"], case["topk"], case["score"], bias=s["bias"], normalize=case["normalize"],
                               factor=_factor(case))
    if op == "route_grad":
        return nuna.route_topk_grad(s["dweights"], s["logits"], s["topk_idx"], case["score"],
                                    normalize=case["normalize"], factor=_factor(case))
    if op == "few":
        return nuna.expert_layer_few(s["x"], s["topk_idx"], s["weights"], s["w1"], s["w1_scale"], s["w2"],
                                     s["w2_scale"], first_expert=s["first"], out=s["out"])
    full = {} if "out" not in s else dict(out=s["out"])
    eight = {} if case["scale"] == "none" else dict(scale=case["scale"], q_out=s["q"], scale_out=s["q_scale"])
    if op == "swiglu":
        nuna.swiglu(s["gu"], offsets=s["offsets"], **full, **eight)
    else:
        nuna.swiglu_grad(s["dout"], s["gu"], offsets=s["offsets"], **full, **eight)
    return tuple(s[name] for name in ("out", "q", "q_scale") if name in s)


def run(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------------------ work

def _f8_bytes(rows, k, scale):
    return rows * (_pad(k, BLOCK) + _pad(k, BLOCK) // BLOCK * (4 if scale == "f32" else 1))


def work(case):
    op, T, es = case["op"], case["tokens"], ESIZE[case["dtype"]]
    if op == "norm":
        n = T * case["hidden"]
        to = n * es + 4 * T if case["scale"] == "none" else _f8_bytes(T, case["hidden"], case["scale"])
        return {"bytes": n * es * (3 if case["residual"] else 1) + to, "flops": (5 if case["residual"] else 4) * n}
    if op == "norm_grad":
        n = T * case["hidden"]
        return {"bytes": n * es * (4 if case["residual"] else 3) + 4 * (T + case["hidden"]), "flops": 9 * n}
    if op == "route":
        n = T * case["experts"]
        return {"bytes": n * es + 8 * T * case["topk"], "flops": 3 * n}
    if op == "route_grad":
        n = T * case["experts"]
        # Where the chosen scores alone are normalised, the others' logits need not be read.
        read = T * case["topk"] if case["normalize"] or case["score"] == "sigmoid" else n
        return {"bytes": (read + n) * es + 8 * T * case["topk"], "flops": 3 * n}
    E, k, count = case["experts"], case["topk"], case["experts"] // case["parts"]
    rows = T * k / case["parts"]  # on average
    if op == "few":
        H, inner = case["hidden"], case["inner"]
        live = count * (1 - (1 - k / E) ** T)  # experts that are reached
        return {"bytes": live * 3 * H * inner + 2 * T * H * es + 8 * T * k, "flops": 6 * rows * H * inner}
    wide = case["inner"] * (2 if op == "swiglu_grad" else 1)
    bytes_ = rows * case["inner"] * es * (3 if op == "swiglu_grad" else 2)
    if case["scale"] == "none" or case["also"]:
        bytes_ += rows * wide * es
    if case["scale"] != "none":
        bytes_ += _f8_bytes(rows, wide, case["scale"])
    return {"bytes": bytes_, "flops": (12 if op == "swiglu_grad" else 6) * rows * case["inner"]}


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_e4m3(v):
    """Float64 values rounded to the nearest e4m3 value, ties to even: 3 bits of fraction from 2^-6 up, steps of 2^-9
    below."""
    e = torch.frexp(v.abs().clamp(min=2.0 ** -20))[1] - 1
    step = torch.exp2(e.clamp(min=-6).double() - 3)
    return torch.round(v / step) * step


def _exact_quantized(x, scale, pitch):
    """x float64 [n, k]: (q values [n, k to a block], scales [n, pitch], ones past the last block)."""
    n, k = x.shape
    v = torch.zeros((n, _pad(k, BLOCK)), dtype=torch.float64, device=x.device)
    v[:, :k] = x
    v = v.view(n, -1, BLOCK)
    s = (v.abs().amax(2) / F8_MAX).clamp(min=SCALE_MIN)
    if scale == "e8m0":
        s = torch.exp2(torch.ceil(torch.log2(s)))
    kept = torch.ones((n, pitch), dtype=torch.float64, device=x.device)
    kept[:, :s.shape[1]] = s
    return _exact_e4m3(v / s.unsqueeze(2)).view(n, -1), kept


def _exact_values(q, scale):
    """Float64 values of a weight matrix [n, k] with a scale per block of 128 x 128."""
    s = scale.double() if scale.dtype == torch.float32 else torch.exp2(scale.view(torch.uint8).double() - 127)
    s = s[:, :q.shape[1] // BLOCK].repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)
    return q.float().double() * s


def _exact_route(s, case):
    z = s["logits"].double()
    alive = torch.isfinite(z)
    key = z
    if s["bias"] is not None:
        key = torch.sigmoid(z) + s["bias"].double()
    # Place of every expert in its row: how many come before it.
    left = torch.where(alive, key, -math.inf)
    picks = []
    for _ in range(case["topk"]):
        best = left.amax(1, keepdim=True)
        first = (left == best).to(torch.uint8).argmax(1, keepdim=True)
        picks.append(torch.where(best > -math.inf, first, -1))
        left = left.scatter(1, first, -math.inf)
    return torch.cat(picks, 1)


def _exact_weights(s, idx, case):
    """(weights [T, k] before the factor, scores of all experts)."""
    z = s["logits"].double()
    p = torch.sigmoid(z) if case["score"] == "sigmoid" else torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
    chosen = torch.where(idx >= 0, p.gather(1, idx.clamp(min=0)), 0.0)
    if case["normalize"]:
        chosen = torch.nan_to_num(chosen / chosen.sum(1, keepdim=True), nan=0.0)
    return chosen, p


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        z = s["x"].double()
        if case["residual"]:
            z = z + s["residual"].double()
        stored = z.to(DTYPES[case["dtype"]]).double()  # what the norm is taken of
        rstd = (stored.square().mean(1, keepdim=True) + EPS).rsqrt()
        y = stored * rstd * s["weight"].double()
        first = (z,) if case["residual"] else ()
        if case["scale"] == "none":
            return (*first, y, rstd.squeeze(1))
        return (*first, *_exact_quantized(y, case["scale"], _pitch(case["hidden"])))
    if op == "norm_grad":
        z, g, r = s["x"].double(), s["dout"].double(), s["rstd"].double().unsqueeze(1)
        u = g * s["weight"].double()
        dx = r * u - z * r ** 3 * (u * z).mean(1, keepdim=True)
        if case["residual"]:
            dx = dx + s["residual"].double()
        return dx, (g * z * r).sum(0)
    if op == "route":
        idx = _exact_route(s, case)
        return idx, _factor(case) * _exact_weights(s, idx, case)[0]
    if op == "route_grad":
        idx, g = s["topk_idx"].long(), s["dweights"].double()
        w, p = _exact_weights(s, idx, case)
        hot = torch.nn.functional.one_hot(idx + 1, case["experts"] + 1)[:, :, 1:].double()  # [T, k, E]
        # The derivative of every chosen weight by every logit, written out: [T, k, E].
        if case["score"] == "softmax":
            jac = w.unsqueeze(2) * (hot - ((w.unsqueeze(2) * hot).sum(1) if case["normalize"] else p).unsqueeze(1))
        elif case["normalize"]:
            slope = (1 - p).unsqueeze(1)  # of the logarithm of a sigmoid
            jac = w.unsqueeze(2) * (hot - (w.unsqueeze(2) * hot).sum(1, keepdim=True)) * slope
        else:
            jac = hot * (p * (1 - p)).unsqueeze(1)
        return _factor(case) * torch.nan_to_num((g.unsqueeze(2) * jac).sum(1), nan=0.0)
    if op == "few":
        H, inner = case["hidden"], case["inner"]
        out = torch.zeros((case["tokens"], H), dtype=torch.float64, device="cuda")
        for e in range(s["experts"]):
            t, j = (s["topk_idx"] == s["first"] + e).nonzero(as_tuple=True)
            if t.numel():
                gu = s["x"][t].double() @ _exact_values(s["w1"][e], s["w1_scale"][e])[:, :H].t()
                h = torch.nn.functional.silu(gu[:, :inner]) * gu[:, inner:]
                y = h @ _exact_values(s["w2"][e], s["w2_scale"][e])[:, :inner].t()
                out.index_add_(0, t, s["weights"][t, j].double().unsqueeze(1) * y)
        return out
    gate, up = s["gu"].double().chunk(2, 1)
    sig = torch.sigmoid(gate)
    v = gate * sig * up
    if op == "swiglu_grad":
        g = s["dout"].double()
        v = torch.cat([g * up * (sig + gate * sig * (1 - sig)), g * gate * sig], 1)
    used = int(s["offsets"][-1])
    v[used:] = 0
    full = (v,) if "out" in s else ()
    if case["scale"] == "none":
        return full
    q, kept = _exact_quantized(v, case["scale"], _pitch(v.shape[1]))
    kept[used:] = 1
    return (*full, q, kept)
