"""The operators of 8-bit layers and of the optimiser step, as timed cases: quantising a matrix with one scale for each
block of 128, the layer's product and its gradients on such operands, and the AdamW step over all tensors of a model.

A case is a dict of plain values; its "kind" says what runs:
  quant     one matrix to 8 bits (rows: a scale for 1 x 128 elements, tiles: for 128 x 128), in one or both directions
  linear    y = x W^T + bias: activations quantised on the way, weights held in 8 bits
  backward  the gradients of that layer: of its input in bf16 and of its weights in fp32
  adamw     one optimiser step over many tensors, moments in 32 or in 8 bits, pruned positions held

Where `own` is false the operators run in their plain form.
"""
import math

import torch

own = False

ROWS, TILES = 0, 1
E4M3 = torch.float8_e4m3fn
E4M3_MAX, LEAST_SCALE = 448.0, 2.0 ** -126


def listed():
    return [
        # the activations of a decode step of eight sequences: latency
        {"name": "quant_decode", "kind": "quant", "R": 8, "C": 4096, "f32": 0, "tiles": 0, "both": 0, "mask": 0},
        # a training batch's activations, kept for both products that read them
        {"name": "quant_train", "kind": "quant", "R": 8192, "C": 4096, "f32": 0, "tiles": 0, "both": 1, "mask": 0},
        # a pruned layer's fp32 master weights, after a step, for the product and its input gradient
        {"name": "quant_weight_pruned", "kind": "quant", "R": 2048, "C": 4608, "f32": 1, "tiles": 1, "both": 1, "mask": 1},
        # one token through a square projection
        {"name": "linear_token", "kind": "linear", "T": 1, "S": 4096, "K": 4096, "f32": 0, "bias": 0},
        # a few sequences' tokens through a wide layer
        {"name": "linear_decode", "kind": "linear", "T": 13, "S": 11008, "K": 4096, "f32": 0, "bias": 0},
        # a short prompt, with nothing a multiple of anything
        {"name": "linear_ragged", "kind": "linear", "T": 333, "S": 1000, "K": 2050, "f32": 0, "bias": 1},
        # a long batch of prompts
        {"name": "linear_prompts", "kind": "linear", "T": 8192, "S": 4096, "K": 4096, "f32": 0, "bias": 0},
        # fine-tuning a narrow layer on a small batch
        {"name": "backward_small", "kind": "backward", "T": 500, "S": 512, "K": 1152},
        # fine-tuning a wide one
        {"name": "backward_large", "kind": "backward", "T": 4096, "S": 4096, "K": 4096},
        # a small head, trained in full precision: launches count
        {"name": "adamw_few", "kind": "adamw", "layers": 1, "d": 192, "w32": 1, "g32": 1, "copy": 0, "bits": 32, "mask": 0, "plan": 0},
        # a pruned model: fp32 master weights with their bf16 copy, bf16 gradients, the mask held
        {"name": "adamw_pruned", "kind": "adamw", "layers": 12, "d": 1024, "w32": 1, "g32": 0, "copy": 1, "bits": 32, "mask": 1, "plan": 0},
        # a larger model whose moments are held in 8 bits
        {"name": "adamw_8bit", "kind": "adamw", "layers": 16, "d": 2048, "w32": 0, "g32": 0, "copy": 0, "bits": 8, "mask": 0, "plan": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: mostly multiples of 128 or 64, some odd ones."""
    n = _log_int(rng, lo, hi)
    step = rng.choice((128, 128, 64, 8, 1))
    return max(step, n // step * step)


def draw(rng):
    kind = rng.choice(("quant", "quant", "linear", "linear", "linear", "backward", "backward", "adamw", "adamw"))
    if kind == "quant":
        tiles = int(rng.random() < 0.4)
        C = _width(rng, 128, 8192)
        R = _width(rng, 128, 8192) if tiles else min(_log_int(rng, 1, 16384), (1 << 25) // C)
        return {"kind": kind, "R": R, "C": C, "f32": int(rng.random() < 0.4), "tiles": tiles, "both": int(rng.random() < 0.6),
                "mask": int(tiles and rng.random() < 0.5)}
    if kind == "linear":
        S, K = _width(rng, 128, 11008), _width(rng, 128, 8192)
        T = min(_log_int(rng, 1, 8192), (1 << 37) // (S * K))
        return {"kind": kind, "T": max(1, T), "S": S, "K": K, "f32": int(rng.random() < 0.25), "bias": int(rng.random() < 0.5)}
    if kind == "backward":
        S, K = _width(rng, 128, 8192), _width(rng, 128, 8192)
        return {"kind": kind, "T": max(1, min(_log_int(rng, 16, 8192), (1 << 36) // (S * K))), "S": S, "K": K}
    w32 = int(rng.random() < 0.6)
    d = _width(rng, 64, 1024)
    return {"kind": kind, "layers": max(1, min(_log_int(rng, 1, 24), (1 << 27) // (13 * d * d))), "d": d, "w32": w32,
            "g32": int(rng.random() < 0.5), "copy": int(w32 and rng.random() < 0.5), "bits": rng.choice((8, 32)),
            "mask": int(rng.random() < 0.4), "plan": rng.randrange(1, 1 << 20)}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(g, T, K, f32):
    """Normal values with a few channels that stand out, as the inputs of a layer have them."""
    x = torch.randn((T, K), generator=g, device="cuda")
    loud = torch.rand(K, generator=g, device="cuda") < 0.005
    x = x * torch.where(loud, 24.0, 1.0)
    return x if f32 else x.to(torch.bfloat16)


def _mask_words(g, S, K, density):
    """Bits of a 2:4 pattern inside kept 64 x 64 blocks: S x ceil(K/32) words, bit k % 32 of word k // 32."""
    words = -(-K // 32)
    nibbles = torch.tensor([3, 5, 6, 9, 10, 12], dtype=torch.int64, device="cuda")
    pick = nibbles[torch.randint(0, 6, (S, words, 8), generator=g, device="cuda")]
    word = (pick << (4 * torch.arange(8, device="cuda"))).sum(-1)
    keep = torch.rand((-(-S // 64), -(-K // 64)), generator=g, device="cuda") < density
    keep = keep.repeat_interleave(64, 0)[:S].repeat_interleave(2, 1)[:, :words]
    word = torch.where(keep, word, torch.zeros_like(word))
    if K % 32:
        word[:, -1] &= (1 << (K % 32)) - 1
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)


def _tensors(case):
    """(rows, columns, whether it is a matrix) of each tensor: per layer four square projections, a gated feed-forward part
    and two norms; an embedding of an odd number of rows."""
    d = case["d"]
    f = d * 11 // 4
    one = [(d, d)] * 4 + [(f, d), (f, d), (d, f)]
    out = [(1003, d, 1)]
    for _ in range(case["layers"]):
        out += [(r, c, 1) for r, c in one] + [(1, d, 0)] * 2
    return out


LR, BETA1, BETA2, EPS, DECAY, STEP, GRAD_SCALE = 1e-4, 0.9, 0.999, 1e-8, 0.01, 1000, 0.5


def _adamw_state(case, g):
    """Flat buffers of weights, gradients and moments, each tensor at a multiple of 128 elements, and its views."""
    parts, at = [], 0
    for r, c, matrix in _tensors(case):
        parts.append((at, r, c, matrix))
        at += -(-r * c // 128) * 128
    wt, gt = (torch.float32 if case[k] else torch.bfloat16 for k in ("w32", "g32"))
    normal = lambda n: torch.randn(n, generator=g, device="cuda")
    st = {"w": (normal(at) * 0.02).to(wt), "g": (normal(at) * 2e-3).to(gt)}
    if case["copy"]:
        st["copy"] = st["w"].to(torch.bfloat16)
    if case["bits"] == 8:
        st["m"], st["v"] = (normal(at) * 100).clamp_(-448, 448).to(E4M3), (normal(at).abs_() * 100 + 0.01).clamp_(max=448).to(E4M3)
        st["ms"], st["vs"] = (torch.rand(at // 128, generator=g, device="cuda") * 1e-5 for _ in range(2))
    else:
        st["m"], st["v"] = normal(at) * 3e-4, (normal(at) * 1e-3).square_()
    views = []
    for at, r, c, matrix in parts:
        t = {k: st[k][at:at + r * c] for k in ("w", "g", "m", "v", "copy") if k in st}
        t |= {k: st[k][at // 128:at // 128 + -(-r * c // 128)] for k in ("ms", "vs") if k in st}
        t["mask"] = _mask_words(g, r, c, 0.6) if case["mask"] and matrix else None
        t["row"], t["decay"] = c, DECAY if matrix else 0.0
        views.append(t)
    st["views"] = views
    return st


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    st = {"case": case}
    if kind == "adamw":
        st |= _adamw_state(case, g)
        if own:
            from paper_2311_14272_amd import adamw
            st["batch"] = adamw.make_batch([adamw.tensor(t["w"], t["g"], t["m"], t["v"], m_scale=t.get("ms"), v_scale=t.get("vs"),
                                                         w_copy=t.get("copy"), mask=t["mask"], row_len=t["row"],
                                                         weight_decay=t["decay"]) for t in st["views"]])
        return st
    if kind == "quant":
        R, C = case["R"], case["C"]
        if case["tiles"]:
            x = torch.randn((R, C), generator=g, device="cuda") * math.sqrt(2.0 / C)
            st["x"] = x if case["f32"] else x.to(torch.bfloat16)
        else:
            st["x"] = _activations(g, R, C, case["f32"])
        st["mask"] = _mask_words(g, R, C, 0.6) if case["mask"] else None
        return st
    T, S, K = case["T"], case["S"], case["K"]
    W = torch.randn((S, K), generator=g, device="cuda") * math.sqrt(2.0 / K)
    if kind == "linear":
        st["x"] = _activations(g, T, K, case["f32"])
        st["w"] = _quant(W, TILES)
        st["bias"] = torch.randn(S, generator=g, device="cuda") if case["bias"] else None
        names = (("w", S, K, TILES),)
    else:
        st["dy"] = (torch.randn((T, S), generator=g, device="cuda") * 1e-3).to(torch.bfloat16)
        st["x_t"] = _quant(_activations(g, T, K, 0).t(), ROWS)
        st["w_t"] = _quant(W.t(), TILES)
        names = (("x_t", K, T, ROWS), ("w_t", K, S, TILES))
    if own:
        from paper_2311_14272_amd import fp8
        for k, rows, cols, how in names:
            st[k] = fp8.Fp8Mat(st[k][0].contiguous(), st[k][1], rows, cols, how)
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------

def _bits(words, C):
    """Mask words as truth values, R x C."""
    bits = (words[:, :, None] >> torch.arange(32, dtype=torch.int32, device=words.device)) & 1
    return bits.reshape(words.shape[0], -1)[:, :C] != 0


def _scale(amax):
    return (amax / torch.full_like(amax, E4M3_MAX)).clamp(min=LEAST_SCALE)


def _quant(x, how):
    """(values, scales): R x round_up(C, 128) in e4m3, zero behind the columns, and fp32 scales, ceil(C/128) x R for rows,
    ceil(R/128) x ceil(C/128) for tiles."""
    R, C = x.shape
    Rb, Cb = -(-R // 128), -(-C // 128)
    x = x.float()
    if how == ROWS:
        x = torch.nn.functional.pad(x, (0, Cb * 128 - C)).view(R, Cb, 128)
        s = _scale(x.abs().amax(2))
        return (x * torch.reciprocal(s)[:, :, None]).to(E4M3).view(R, Cb * 128), s.t().contiguous()
    x = torch.nn.functional.pad(x, (0, Cb * 128 - C, 0, Rb * 128 - R)).view(Rb, 128, Cb, 128)
    s = _scale(x.abs().amax((1, 3)))
    return (x * torch.reciprocal(s)[:, None, :, None]).to(E4M3).view(Rb * 128, Cb * 128)[:R].contiguous(), s


def _values(q, s, how):
    """The fp32 values that 8-bit operands stand for."""
    R, C = q.shape
    v = q.float()
    if how == ROWS:
        return (v.view(R, C // 128, 128) * s.t()[:, :, None]).view(R, C)
    return v * s.repeat_interleave(128, 0)[:R].repeat_interleave(128, 1)


def _product(x, w, x_how, w_how):
    return _values(*x, x_how) @ _values(*w, w_how).t()


def _adamw(t, bits):
    """One tensor's step, in place."""
    w, gr = t["w"].float(), t["g"].float() * GRAD_SCALE
    n = w.numel()
    if bits == 8:
        spread = lambda s: s.repeat_interleave(128)[:n]
        m, u = t["m"].float() * spread(t["ms"]), t["v"].float() * spread(t["vs"])
        v = u * u
    else:
        m, v = t["m"], t["v"]
    if t["mask"] is not None:
        kept = _bits(t["mask"], t["row"]).reshape(-1)
        gr, m, v = (torch.where(kept, a, torch.zeros_like(a)) for a in (gr, m, v))
    m = m * BETA1 + gr * (1 - BETA1)
    v = v * BETA2 + (gr * gr) * (1 - BETA2)
    u = torch.sqrt(v)
    new = w * (1 - LR * t["decay"]) - (m / (u * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS)) * (LR / (1 - BETA1 ** STEP))
    if t["mask"] is not None:
        new = torch.where(kept, new, w)
    t["w"].copy_(new)
    if "copy" in t:
        t["copy"].copy_(new)
    if bits == 32:
        t["m"].copy_(m)
        t["v"].copy_(v)
        return
    blocks = lambda a: torch.nn.functional.pad(a, (0, -n % 128)).view(-1, 128)
    m, u = blocks(m), blocks(u)
    ms, us = _scale(m.abs().amax(1)), _scale(u.amax(1))
    qm, qu = (m * torch.reciprocal(ms)[:, None]).to(E4M3), u * torch.reciprocal(us)[:, None]
    qu = torch.where(u > 0, qu.clamp(min=2.0 ** -9), qu).to(E4M3)   # a moment that is not zero stays so
    t["m"].copy_(qm.view(-1)[:n])
    t["v"].copy_(qu.view(-1)[:n])
    t["ms"].copy_(ms)
    t["vs"].copy_(us)


def _state_out(st):
    return {k: st[k] for k in ("w", "m", "v", "ms", "vs", "copy") if k in st}


def run(st):
    case = st["case"]
    kind = case["kind"]
    if kind == "quant":
        how = TILES if case["tiles"] else ROWS
        if own:
            from paper_2311_14272_amd import fp8
            if case["both"]:
                return [(a.q, a.scale) for a in fp8.quantize_both(st["x"], how, mask=st["mask"])]
            a = fp8.quantize(st["x"], how, mask=st["mask"])
            return [(a.q, a.scale)]
        x = st["x"]
        if st["mask"] is not None:
            x = torch.where(_bits(st["mask"], case["C"]), x, torch.zeros_like(x))
        return [_quant(a, how) for a in ((x, x.t()) if case["both"] else (x,))]
    if kind == "linear":
        if own:
            from paper_2311_14272_amd import fp8
            return fp8.linear(st["x"], st["w"], bias=st["bias"])
        y = _product(_quant(st["x"], ROWS), st["w"], ROWS, TILES)
        return (y if st["bias"] is None else y + st["bias"]).to(torch.bfloat16)
    if kind == "backward":
        if own:
            from paper_2311_14272_amd import fp8
            return fp8.linear_backward(st["dy"], st["x_t"], st["w_t"])
        dx = _product(_quant(st["dy"], ROWS), st["w_t"], ROWS, TILES)
        dw = _product(_quant(st["dy"].t(), ROWS), st["x_t"], ROWS, ROWS)
        return dx.to(torch.bfloat16), dw
    if own:
        from paper_2311_14272_amd import adamw
        adamw.step(st["batch"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=STEP, grad_scale=GRAD_SCALE)
    else:
        [_adamw(t, case["bits"]) for t in st["views"]]
    return _state_out(st)


def work(case):
    kind = case["kind"]
    if kind == "quant":
        n = case["R"] * case["C"]
        scales = n / 128 / (128 if case["tiles"] else 1) * 4
        return {"bytes": n * (4 if case["f32"] else 2) + (1 + case["both"]) * (n + scales) + n / 8 * case["mask"], "flops": 2 * n}
    if kind == "adamw":
        total = 0.0
        for r, c, matrix in _tensors(case):
            w, gr, mv = (4 if case["w32"] else 2), (4 if case["g32"] else 2), (8 if case["bits"] == 32 else 2)
            kept = 0.5 * 0.6 if case["mask"] and matrix else 1.0
            each = kept * (2 * w + gr + mv + 2 * case["copy"]) + mv
            each += 16 / 128 if case["bits"] == 8 else 0
            total += r * c * (each + (1 / 8 if kept < 1 else 0))
        return {"bytes": total, "flops": 14 * sum(r * c for r, c, _ in _tensors(case))}
    T, S, K = case["T"], case["S"], case["K"]
    if kind == "linear":
        return {"bytes": T * K * (4 if case["f32"] else 2) + S * K * (1 + 4 / 16384) + T * S * 2 + S * 4 * case["bias"], "flops": 2 * T * S * K}
    return {"bytes": T * S * 2 + S * K * (1 + 4 / 16384) + T * K * (1 + 4 / 128) + T * K * 2 + S * K * 4, "flops": 4 * T * S * K}


# ---- the definition in 64 bits --------------------------------------------------------------------------------
# The scales and the value that is rounded to 8 bits are fp32 numbers by definition; everything else is not rounded.

def _exact_scale(amax):
    return torch.maximum((amax / torch.full_like(amax, E4M3_MAX)).float().double(), torch.full_like(amax, LEAST_SCALE))


def _exact_codes(x, s):
    """e4m3 values of x / s for scales s of x's shape."""
    inverse = (torch.ones_like(s) / s).float().double()
    return (x * inverse).float().to(E4M3).double()


def _exact_quant(x, how, keep=None):
    x = x.double()
    if keep is not None:
        x = torch.where(keep, x, torch.zeros_like(x))
    R, C = x.shape
    Rb, Cb = (R + 127) // 128, (C + 127) // 128
    full = torch.zeros((Rb * 128, Cb * 128), dtype=torch.float64, device=x.device)
    full[:R, :C] = x
    a = full.abs().reshape(Rb * 128, Cb, 128).amax(-1)
    if how == TILES:
        a = a.reshape(Rb, 128, Cb).amax(1)
        s = _exact_scale(a)
        each = s.repeat_interleave(128, 0).repeat_interleave(128, 1)
        return _exact_codes(full, each)[:R], s, each[:R]
    s = _exact_scale(a)
    each = s.repeat_interleave(128, 1)
    return _exact_codes(full, each)[:R], s[:R].t().contiguous(), each[:R]


def _exact_held(h, how):
    q, s = (h.q, h.scale) if hasattr(h, "q") else h
    q, s = q.double(), s.double()
    if how == ROWS:
        return q * s.t().repeat_interleave(128, 1)
    return q * s.repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)


def _exact_adamw(st, case):
    out = {k: v.double() for k, v in _state_out(st).items()}
    at = 0
    for t in st["views"]:
        n = t["w"].numel()
        here, nb = slice(at, at + n), (n + 127) // 128
        blocks = slice(at // 128, at // 128 + nb)
        w, gr, m, v = (t[k].double() for k in ("w", "g", "m", "v"))
        gr = gr * GRAD_SCALE
        if case["bits"] == 8:
            m = m * t["ms"].double().repeat_interleave(128)[:n]
            v = (v * t["vs"].double().repeat_interleave(128)[:n]) ** 2
        keep = torch.ones(n, dtype=torch.bool, device=w.device)
        if t["mask"] is not None:
            k = torch.arange(t["row"], device=w.device)
            keep = ((t["mask"][:, k // 32].long() >> (k % 32)) & 1).bool().reshape(-1)
        m = torch.where(keep, BETA1 * m + (1 - BETA1) * gr, 0.0)
        v = torch.where(keep, BETA2 * v + (1 - BETA2) * gr ** 2, 0.0)
        hat = (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
        w = torch.where(keep, w - LR * t["decay"] * w - LR * hat, w)
        out["w"][here] = w
        if "copy" in out:
            out["copy"][here] = w
        if case["bits"] == 32:
            out["m"][here], out["v"][here] = m, v
        else:
            for name, scale, a in (("m", "ms", m), ("v", "vs", v.sqrt())):
                full = torch.zeros(nb * 128, dtype=torch.float64, device=w.device)
                full[:n] = a
                s = _exact_scale(full.reshape(nb, 128).abs().amax(1))
                q = _exact_codes(full, s.repeat_interleave(128))
                if name == "v":
                    q = torch.where((full > 0) & (q == 0), 2.0 ** -9, q)
                out[name][here], out[scale][blocks] = q[:n], s
        at += nb * 128
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "adamw":
        return _exact_adamw(st, case)
    if kind == "quant":
        how = TILES if case["tiles"] else ROWS
        C = case["C"]
        keep = None
        if st["mask"] is not None:
            k = torch.arange(C, device="cuda")
            keep = ((st["mask"][:, k // 32].long() >> (k % 32)) & 1).bool()
        out = [_exact_quant(st["x"], how, keep)[:2]]
        if case["both"]:
            out.append(_exact_quant(st["x"].t(), how, None if keep is None else keep.t())[:2])
        return out
    if kind == "linear":
        q, _, each = _exact_quant(st["x"], ROWS)
        y = torch.mm(q * each, _exact_held(st["w"], TILES).t())
        return y if st["bias"] is None else y + st["bias"].double()
    q, _, each = _exact_quant(st["dy"], ROWS)
    dx = torch.mm(q * each, _exact_held(st["w_t"], TILES).t())
    q, _, each = _exact_quant(st["dy"].t(), ROWS)
    dw = torch.mm(q * each, _exact_held(st["x_t"], ROWS).t())
    return dx, dw
