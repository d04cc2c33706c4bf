"""The operators around the double-pruned 2:4 layer, as measurable cases: the norm in front of it with its gradient, the
layer's product on 8-bit operands, and the optimizer step behind its gradients.

Kinds of a case:

  norm      residual addition and RMS norm of b tokens of width d: bf16 output with the row statistics for training, or 8-bit
            output with a scale per token for the 8-bit product
  norm_bwd  its gradient: dx (with the residual stream's own gradient added) and the norm weight's gradient
  product   Y = X (W^R)^T on e4m3 operands with a scale per token and per weight row, optionally plus a bf16 term
  update    AdamW over the tensors of some transformer blocks whose linear layers are packed 2:4; 32-bit states come with the
            global gradient norm, clipping and the skip of a step that is not finite, 8-bit states (e4m3 with a scale per
            128 elements) with a gradient scale known beforehand

Widths are those of the layer sets of `paper_2405_16325_amd/inputs.py`, of the tests' ragged layers, or numbers between them.
With `own` false the same results come from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

BF16, F32, F8, U8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn, torch.uint8
EPS = 1e-5
BLOCK, F8_MAX, TINY = 128, 448.0, 1e-30
LR, BETA1, BETA2, ADAM_EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
INV_SCALE, MAX_NORM = 1.0 / 1024.0, 1.0


# ------------------------------------------------------------------------------------------------------------- the cases

def _norm(name, b, d, residual, q8):
    return {"name": name, "kind": "norm", "b": b, "d": d, "residual": residual, "q8": q8}


def _norm_bwd(name, b, d, residual):
    return {"name": name, "kind": "norm_bwd", "b": b, "d": d, "residual": residual}


def _product(name, b, d_out, d_in, add):
    return {"name": name, "kind": "product", "b": b, "d_out": d_out, "d_in": d_in, "add": add}


def _update(name, bits, width, blocks, rank, packed, odd, master, grad_bits):
    return {"name": name, "kind": "update", "bits": bits, "width": width, "blocks": blocks, "rank": rank, "packed": packed,
            "odd": odd, "master": master, "grad_bits": grad_bits}


def listed():
    return [
        # one token in front of the smallest layer, 8-bit output: latency
        _norm("norm_token", 1, 768, True, True),
        # the largest training batch
        _norm("norm_train", 16384, 9216, True, False),
        # a prompt of odd length in front of the 8-bit product
        _norm("norm_prompt_q8", 777, 5120, True, True),
        # the largest training batch's gradient, residual stream included
        _norm_bwd("norm_bwd_train", 16384, 9216, True),
        # a micro-batch on a width that is a multiple of 8 only
        _norm_bwd("norm_bwd_ragged", 1000, 1000, False),
        # one token through a large layer: a single pass over the packed 8-bit weight
        _product("q8_token", 1, 36864, 9216, False),
        # a prompt of odd length, the residual stream added in the same call
        _product("q8_prompt", 777, 20480, 5120, True),
        # prefill of many prompts through the largest layer
        _product("q8_prefill", 8192, 36864, 9216, False),
        # adapters, norms and biases of two small blocks, whose weights are frozen: many small tensors, latency
        _update("update_adapters", 32, 768, 2, 32, False, 1, True, 32),
        # one ordinary block, packed values with fp32 masters
        _update("update_block", 32, 5120, 1, 0, True, 0, True, 16),
        # four small blocks and a tensor of odd length, 8-bit states
        _update("update8_blocks", 8, 2560, 4, 0, True, 50257, True, 16),
        # the largest block, 8-bit states, bf16 weights only
        _update("update8_large", 8, 9216, 1, 128, True, 0, False, 16),
    ]


def _log_uniform(rng, lo, hi):
    return lo * (hi / lo) ** rng.random()


def _width(rng, lo, hi, quantum):
    w = int(_log_uniform(rng, lo, hi) / quantum + 0.5) * quantum
    return max(quantum, min(w, hi // quantum * quantum))


def _elements(case):
    return sum(n for n, _ in _tensors(case))


def draw(rng):
    """One more case: kinds, token counts, widths and tensor sets over the ranges the listed cases span."""
    kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "product", "product", "product", "update", "update", "update"])
    q = rng.choices([256, 64, 8], [4, 3, 3])[0]
    if kind in ("norm", "norm_bwd"):
        d = _width(rng, 64, 36864 if q == 256 else 9216, q)
        b = int(_log_uniform(rng, 1, 16384) + 0.5)
        b = max(1, min(b, 16384 * 9216 // d))
        c = _norm("", b, d, rng.random() < 0.7, rng.random() < 0.5) if kind == "norm" else _norm_bwd("", b, d, rng.random() < 0.7)
    elif kind == "product":
        lo, hi = (512, 36864) if q == 256 else (512, 9216) if q == 64 else (200, 2056)
        d_out, d_in = _width(rng, lo, hi, q), _width(rng, lo, hi, q)
        b = int(_log_uniform(rng, 1, 8192 if q >= 64 else 2048) + 0.5)
        b = max(1, min(b, 8192 * 36864 * 9216 // (d_out * d_in)))
        c = _product("", b, d_out, d_in, rng.random() < 0.4)
    else:
        bits, packed = rng.choice([8, 32]), rng.random() < 0.7
        width = _width(rng, 128, 9216, rng.choice([256, 64, 8]))
        rank = rng.choice([0, 32, 64, 128])
        odd, master, grad_bits = rng.choice([0, 1, int(_log_uniform(rng, 2, 100000))]), rng.random() < 0.6, rng.choice([16, 16, 32])
        c = _update("", bits, width, 1, rank, packed, odd, master, grad_bits)
        most = 500_000_000 if bits == 8 else 157_000_000
        c["blocks"] = int(_log_uniform(rng, 1, max(1.0, min(12.0, most / _elements(c)))) + 0.5)
        while c["blocks"] > 1 and _elements(c) > most:
            c["blocks"] -= 1
        if _elements(c) > most:
            c["width"] = 5120 if bits == 32 else 9216 - 256
    del c["name"]
    return c


def _tensors(case):
    """(elements, weight decay) of each tensor: packed values of q, k, v, o, fc1, fc2, their adapters, biases, two norms."""
    w, r, got = case["width"], case["rank"], []
    for _ in range(case["blocks"]):
        for d_out, d_in in ((w, w), (w, w), (w, w), (w, w), (4 * w, w), (w, 4 * w)):
            if case["packed"]:
                got.append((d_out * d_in // 2, DECAY))
            if r:
                got += [(d_in * r, DECAY), (r * d_out, DECAY)]
            got.append((d_out, 0.0))
        got += [(w, 0.0), (w, 0.0)]
    if case["odd"]:
        got.append((case["odd"], DECAY))
    return got


# ------------------------------------------------------------------------------------------------------------ the inputs

def _pruned(vals):
    """Packed 2:4 form of a weight: (values bf16[d_out, d_in/2], index bytes u8[d_out, d_in/8])."""
    d_out, d_in = vals.shape
    a = vals.abs().view(d_out, d_in // 4, 4)
    beats = lambda i, j: a[..., j] > a[..., i] if j > i else a[..., j] >= a[..., i]      # noqa: E731
    keep = torch.stack([sum(beats(i, j).to(U8) for j in range(4) if j != i) < 2 for i in range(4)], dim=-1)
    first = keep.to(U8).argmax(-1)
    last = 3 - keep.flip(-1).to(U8).argmax(-1)
    at = torch.stack([first, last], dim=-1)
    kept = torch.gather(vals.view(d_out, d_in // 4, 4), 2, at).reshape(d_out, d_in // 2)
    nibble = (first | (last << 2)).to(U8).view(d_out, d_in // 8, 2)
    return kept, (nibble[..., 0] | (nibble[..., 1] << 4)).contiguous()


def _rows_to_8_bits(x):
    """x -> (e4m3 codes, fp32 scale per row)."""
    amax = x.abs().amax(1)
    scale = torch.where(amax < TINY, 0.0, amax * (1.0 / F8_MAX))
    inv = torch.where(amax < TINY, 0.0, amax.reciprocal() * F8_MAX)
    return (x * inv[:, None]).clamp(-F8_MAX, F8_MAX).to(F8), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def gauss(shape, std, dtype=BF16):
        return torch.randn(shape, generator=gen, device="cuda", dtype=F32).mul_(std).to(dtype)

    kind = case["kind"]
    if kind == "norm":
        b, d = case["b"], case["d"]
        return {"kind": kind, "q8": case["q8"], "x": gauss((b, d), 1.0),
                "res": gauss((b, d), 2.0) if case["residual"] else None, "w": (1.0 + gauss((d,), 0.1, F32)).to(BF16)}
    if kind == "norm_bwd":
        b, d = case["b"], case["d"]
        h = gauss((b, d), 2.0)
        rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
        return {"kind": kind, "dy": gauss((b, d), 1e-3), "h": h, "rstd": rstd, "w": (1.0 + gauss((d,), 0.1, F32)).to(BF16),
                "dh": gauss((b, d), 1e-3) if case["residual"] else None}
    if kind == "product":
        b, d_out, d_in = case["b"], case["d_out"], case["d_in"]
        vals, meta = _pruned(gauss((d_out, d_in), 0.02))
        wq, wscale = _rows_to_8_bits(vals.float())
        q, scale = _rows_to_8_bits(gauss((b, d_in), 1.0, F32))
        return {"kind": kind, "q": q, "scale": scale, "wq": wq, "wscale": wscale, "meta": meta,
                "add": gauss((b, d_out), 1.0) if case["add"] else None}

    # every tensor of a set starts at a multiple of 128 elements of one allocation; the gaps hold zeros
    sizes = _tensors(case)
    starts, total = [], 0
    for n, _ in sizes:
        starts.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    lens = torch.tensor([n for n, _ in sizes], device="cuda")
    padded = (lens + BLOCK - 1) // BLOCK * BLOCK
    start = torch.tensor(starts, device="cuda").repeat_interleave(padded, output_size=total)
    index = torch.arange(total, device="cuda").sub_(start)
    inside = index < lens.repeat_interleave(padded, output_size=total)
    gdtype = F32 if case["grad_bits"] == 32 else BF16
    st = {"kind": kind, "bits": case["bits"], "step": 100, "sizes": sizes, "starts": starts,
          "grad": gauss((total,), 0.5, gdtype) * inside,
          "index": index.to(torch.int32), "decay": torch.tensor([x for _, x in sizes], device="cuda", dtype=F32).repeat_interleave(
              padded // BLOCK, output_size=total // BLOCK), "master": None, "m_scale": None, "v_scale": None}
    del start, index
    p = gauss((total,), 0.02, F32) * inside
    st["param"] = p.to(BF16)
    if case["master"]:
        st["master"] = p
    m, v = gauss((total,), 1e-4, F32) * inside, gauss((total,), 5e-4, F32).square_() * inside
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
        st["control"] = torch.tensor([0.0, 0.0, 99.0, 0.0], device="cuda")
    else:
        mq, st["m_scale"] = _rows_to_8_bits(m.view(-1, BLOCK))
        rq, st["v_scale"] = _rows_to_8_bits(v.sqrt().view(-1, BLOCK))
        st["m"], st["v"] = mq.view(-1), rq.view(-1)
        st["control"] = None
    if own:
        from paper_2405_16325_amd import binding as sl
        cut = lambda t: [t[s:s + n] for s, (n, _) in zip(starts, sizes)] if t is not None else None         # noqa: E731
        tiles = lambda t: [t[s // BLOCK:(s + n + BLOCK - 1) // BLOCK] for s, (n, _) in zip(starts, sizes)] if t is not None else None  # noqa: E731
        st["plan"] = sl.slope_adamw_plan(cut(st["param"]), cut(st["grad"]), cut(st["m"]), cut(st["v"]), masters=cut(st["master"]),
                                         m_scales=tiles(st["m_scale"]), v_scales=tiles(st["v_scale"]),
                                         weight_decay=[x for _, x in sizes])
    return st


# -------------------------------------------------------------------------------------------------------- the plain forms

def _plain_norm(s):
    h = s["x"] if s["res"] is None else (s["x"].float() + s["res"].float()).to(BF16)
    hf = h.float()
    rstd = torch.rsqrt(hf.square().mean(1) + EPS)
    y = hf * rstd[:, None] * s["w"].float()
    got = {} if s["res"] is None else {"h": h}
    if s["q8"]:
        got["q"], got["scale"] = _rows_to_8_bits(y)
    else:
        got["y"], got["rstd"] = y.to(BF16), rstd
    return got


def _plain_norm_bwd(s):
    dy, xh = s["dy"].float(), s["h"].float() * s["rstd"][:, None]
    g = dy * s["w"].float()
    dx = (g - xh * (g * xh).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(BF16), "dw": (dy * xh).sum(0).to(BF16)}


def _positions(meta):
    """Column of each packed value: int64[d_out, d_in/2]."""
    d_out, bytes_ = meta.shape
    m = meta.to(torch.int64)
    idx = torch.stack([m & 3, (m >> 2) & 3, ((m >> 4) & 3) + 4, (m >> 6) + 4], dim=-1)
    return (idx + 8 * torch.arange(bytes_, device=meta.device)[:, None]).view(d_out, -1)


def _plain_product(s):
    d_out, half = s["wq"].shape
    w = torch.zeros((d_out, 2 * half), device="cuda", dtype=F32)
    w.scatter_(1, _positions(s["meta"]), s["wq"].float() * s["wscale"][:, None])
    y = torch.matmul(s["q"].float() * s["scale"][:, None], w.t())
    return (y if s["add"] is None else y + s["add"].float()).to(BF16)


def _plain_round(x, u):
    """x in [0, 448] to a neighbour in e4m3: up with the probability (for evenly spread u) of its distance from the lower one."""
    e = (torch.frexp(x).exponent - 1).clamp_(min=-6)
    ulp = torch.ldexp(torch.ones_like(x), e - 3)
    low = torch.where(x < 2.0 ** -6, 8.0, 0.0)
    return (torch.floor(x / ulp + low + u) - low) * ulp


def _plain_store(x, u, root):
    """Blocks of 128 of x -> (e4m3 codes, scales); a root that is not zero does not become zero."""
    a = x.view(-1, BLOCK).abs()
    amax = a.amax(1, keepdim=True)
    scale = torch.where(amax < TINY, 0.0, amax * (1.0 / F8_MAX))
    inv = torch.where(amax < TINY, 0.0, amax.reciprocal() * F8_MAX)
    a = (a * inv).clamp_(max=F8_MAX)
    q = _plain_round(a, u.view(-1, BLOCK))
    if root:
        q = torch.where((a > 0) & (q == 0), 2.0 ** -9, q)
    return torch.copysign(q, x.view(-1, BLOCK)).to(F8).view(-1), scale.view(-1)


def _plain_update(s):
    t, bits = s["step"], s["bits"]
    skip = None
    if s["control"] is not None:
        control = s["control"]
        norm = s["grad"].float().square().sum().sqrt() * INV_SCALE
        fine = torch.isfinite(norm)
        skip = ~fine
        coef = torch.where(fine, INV_SCALE * torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0), 0.0)
        control[0], control[1] = norm, coef
        control[2] += fine.to(F32)
        t = control[2]
        bc1, bc2 = -torch.expm1(t * math.log(BETA1)), -torch.expm1(t * math.log(BETA2))
        root2 = bc2.sqrt()
    else:
        coef = INV_SCALE
        bc1, bc2 = 1.0 - BETA1 ** t, 1.0 - BETA2 ** t
        root2 = math.sqrt(bc2)
    g = s["grad"].float() * coef
    if bits == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        v = v * v
    m2 = m * BETA1 + g * (1.0 - BETA1)
    v2 = v * BETA2 + g * g * (1.0 - BETA2)
    r2 = v2.sqrt()
    p = (s["param"].float() if s["master"] is None else s["master"]).view(-1, BLOCK)
    p2 = (p * (1.0 - LR * s["decay"])[:, None]).view(-1) - (LR / bc1) * (m2 / (r2 / root2 + ADAM_EPS))
    if skip is not None:
        p2, m2, v2 = torch.where(skip, p.view(-1), p2), torch.where(skip, m, m2), torch.where(skip, v, v2)
    if s["master"] is not None:
        s["master"].copy_(p2)
    s["param"].copy_(p2)
    if bits == 32:
        m.copy_(m2)
        v.copy_(v2)
    else:
        h = (s["index"].to(torch.int64) * 0x6A09E667 + t * 0x9E3779B9) & 0xFFFFFFFF
        u = (h >> 12).float() * 2.0 ** -20
        mq, ms = _plain_store(m2, u, False)
        u = ((h ^ 0x80000000) >> 12).float() * 2.0 ** -20
        rq, rs = _plain_store(r2, u, True)
        s["m"].view(U8).copy_(mq.view(U8))
        s["v"].view(U8).copy_(rq.view(U8))
        s["m_scale"].copy_(ms)
        s["v_scale"].copy_(rs)


def _updated(s):
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale", "control")}


# -------------------------------------------------------------------------------------------------------------- one pass

def run(state):
    s, kind = state, state["kind"]
    if not own:
        if kind == "update":
            _plain_update(s)
            return _updated(s)
        return {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "product": _plain_product}[kind](s)
    from paper_2405_16325_amd import binding as sl
    if kind == "norm":
        y, h, rstd, q, scale = sl.slope_rmsnorm_fwd(s["x"], s["w"], EPS, residual=s["res"], want_y=not s["q8"],
                                                    want_rstd=not s["q8"], want_q8=s["q8"])
        got = {} if s["res"] is None else {"h": h}
        got.update({"q": q, "scale": scale} if s["q8"] else {"y": y, "rstd": rstd})
        return got
    if kind == "norm_bwd":
        dx, dw = sl.slope_rmsnorm_bwd(s["dy"], s["h"], s["w"], s["rstd"], dh=s["dh"])
        return {"dx": dx, "dw": dw}
    if kind == "product":
        return sl.slope_spmm_fwd_q8(s["q"], s["scale"], s["wq"], s["meta"], s["wscale"], add=s["add"])
    if s["control"] is not None:
        sl.slope_grad_norm(s["plan"], s["control"], INV_SCALE, MAX_NORM)
        sl.slope_adamw_step(s["plan"], LR, BETA1, BETA2, ADAM_EPS, control=s["control"])
    else:
        sl.slope_adamw_step(s["plan"], LR, BETA1, BETA2, ADAM_EPS, step=s["step"], grad_scale=INV_SCALE)
    return _updated(s)


def work(case):
    """Each input read once, each output written once.  The 2:4 product executes half of the dense multiply-adds."""
    kind = case["kind"]
    if kind == "norm":
        b, d = case["b"], case["d"]
        moved = 2 * b * d * (3 if case["residual"] else 1) + 2 * d + (b * d if case["q8"] else 2 * b * d) + 4 * b
        return {"bytes": moved, "flops": 6 * b * d}
    if kind == "norm_bwd":
        b, d = case["b"], case["d"]
        return {"bytes": 2 * b * d * (4 if case["residual"] else 3) + 4 * b + 4 * d, "flops": 11 * b * d}
    if kind == "product":
        b, d_out, d_in = case["b"], case["d_out"], case["d_in"]
        return {"bytes": b * d_in + 4 * b + d_out * d_in * 5 // 8 + 4 * d_out + 2 * b * d_out * (2 if case["add"] else 1),
                "flops": b * d_out * d_in}
    n = _elements(case)
    each = case["grad_bits"] / 8 + (2 + 8 if case["master"] else 4) + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)
    return {"bytes": n * each, "flops": 20 * n}


# ------------------------------------------------------------------------------------------------- the definition in fp64

def exact(case, seed):
    """The definitions in 64 bits.  Values held in 8 bits stand here as they are before that rounding."""
    s, kind = prepare(case, seed), case["kind"]
    f = lambda t: t.to(torch.float64)                                                        # noqa: E731
    if kind == "norm":
        h = f(s["x"])
        got = {}
        if s["res"] is not None:
            h = h + f(s["res"])
            got["h"] = h
            h = f(h.to(BF16))                   # the statistics are those of the stream as it is stored
        rstd = (h.pow(2).sum(1) / case["d"] + EPS) ** -0.5
        y = h * rstd[:, None] * f(s["w"])
        if not case["q8"]:
            return {**got, "y": y, "rstd": rstd}
        top = y.abs().max(1).values
        return {**got, "q": y * 448 / top[:, None], "scale": top / 448}
    if kind == "norm_bwd":
        # y_j = h_j w_j r(h): dx = r (w dy) - h r^3 sum(w dy h) / d
        dy, h, r = f(s["dy"]), f(s["h"]), f(s["rstd"])
        t = dy * f(s["w"])
        dx = r[:, None] * t - h * (r ** 3 * (t * h).sum(1) / case["d"])[:, None]
        if s["dh"] is not None:
            dx += f(s["dh"])
        return {"dx": dx, "dw": torch.mv((dy * h).t(), r)}
    if kind == "product":
        meta, wq = s["meta"], f(s["wq"])
        w = torch.zeros((case["d_out"], case["d_in"]), dtype=torch.float64, device="cuda")
        for slot in range(4):                   # value 4 i + slot of a row lies in the group 2 i + slot / 2
            col = (meta >> (2 * slot) & 3).long() + 4 * (slot // 2)
            col += torch.arange(0, case["d_in"], 8, device="cuda")
            w.scatter_(1, col, wq[:, slot::4])
        y = torch.mm(f(s["q"]), w.t().contiguous())
        y *= f(s["scale"])[:, None]
        y *= f(s["wscale"])
        return y if s["add"] is None else y.add_(f(s["add"]))
    n = s["grad"].numel()
    spread = lambda x: f(x).repeat_interleave(BLOCK, output_size=n)                          # noqa: E731
    c, t, control = INV_SCALE, s["step"], None
    if s["control"] is not None:
        norm = float(torch.linalg.vector_norm(f(s["grad"]))) * INV_SCALE
        c = INV_SCALE * min(1.0, MAX_NORM / (norm + 1e-6))
        control = torch.tensor([norm, c, t, 0.0], dtype=torch.float64)
    g = f(s["grad"]) * c
    m, v = f(s["m"]), f(s["v"])
    if s["bits"] == 8:
        m, v = m * spread(s["m_scale"]), (v * spread(s["v_scale"])) ** 2
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
    p = f(s["param"]) if s["master"] is None else f(s["master"])
    p = p - LR * spread(s["decay"]) * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + ADAM_EPS)
    got = {"param": p, "master": None if s["master"] is None else p, "m": m, "v": v, "m_scale": None, "v_scale": None,
           "control": control}
    if s["bits"] == 8:
        r = v ** 0.5
        for name, x in (("m", m), ("v", r)):
            top = x.view(-1, BLOCK).abs().max(1).values
            got[name + "_scale"] = top / 448
            got[name] = torch.where(spread(top) > 0, x / spread(top).clamp(min=1e-300) * 448, 0.0)
    return got
