"""What the training operators next to the few-bit activations are measured on.

Three families, each with its plain form (elementary torch operations in 32 bits) and the library's kernels:

* attention, forward and backward (the backward pass recomputes the probabilities from the saved row statistics),
  on dense (batch, length, heads, head_dim) tensors or on sequences of unequal length packed one after the other;
* the RMS norm of every query and key head with the position rotation in the same pass, forward and backward;
* one AdamW step over all tensors of a model, moments in 32 bits or in 8 (float8 codes with one binary32 scale per
  256 elements, rounded stochastically from a counter-based generator whose seed is an input).
"""
import math

import torch

own = False

BLOCK = 256                      # elements of an 8-bit moment that share one scale
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def _attn(name, op, dtype, batch, q_len, k_len, heads, kv_heads, head_dim, causal, fused=False, docs=0):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "q_len": q_len, "k_len": k_len, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "fused": fused, "docs": docs}


def _qk(name, op, dtype, batch, length, heads, kv_heads, head_dim, rotary_dim, interleaved, positions):
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "length": length, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "rotary_dim": rotary_dim, "interleaved": interleaved,
            "positions": positions}


def _adamw(name, dtype, state_bits, master, layers, width, vocab, odd):
    return {"name": name, "op": "adamw", "dtype": dtype, "state_bits": state_bits, "master": master, "layers": layers,
            "width": width, "vocab": vocab, "odd": odd}


def listed():
    return [
        # a short sequence of a small encoder: fewer tiles than SMs, the call's latency counts
        _attn("attn_fwd_short_f16", "attention_fwd", "f16", 2, 77, 77, 4, 4, 64, False),
        # long-context pre-training: causal, four query heads share a key head, read out of one fused projection
        _attn("attn_fwd_long_bf16", "attention_fwd", "bf16", 1, 16384, 16384, 8, 2, 128, True, fused=True),
        # fine-tuning on a few short documents packed into one row, odd lengths
        _attn("attn_bwd_packed_f16", "attention_bwd", "f16", 1, 1500, 1500, 6, 2, 64, True, docs=9),
        # a pre-training micro-batch
        _attn("attn_bwd_train_bf16", "attention_bwd", "bf16", 4, 2048, 2048, 16, 4, 128, True),
        # long-context pre-training, the backward pass of the forward case above
        _attn("attn_bwd_long_bf16", "attention_bwd", "bf16", 1, 16384, 16384, 8, 2, 128, True, fused=True),
        # a handful of tokens: latency
        _qk("qk_fwd_few_f32", "qk_fwd", "f32", 1, 5, 8, 2, 64, 64, False, True),
        # a training micro-batch of long rows, views of one fused projection
        _qk("qk_fwd_train_bf16", "qk_fwd", "bf16", 4, 8192, 32, 8, 128, 128, False, False),
        # backward of a small odd batch, rotation of part of each head, neighbouring pairs
        _qk("qk_bwd_odd_f16", "qk_bwd", "f16", 3, 333, 12, 4, 80, 40, True, True),
        # backward of the training micro-batch
        _qk("qk_bwd_train_bf16", "qk_bwd", "bf16", 4, 8192, 32, 8, 128, 128, False, False),
        # an adapter's few odd-sized tensors, 8-bit moments: latency
        _adamw("adamw8_small_f32", "f32", 8, False, 1, 40, 0, True),
        # a model of some forty million parameters trained in binary32, ordinary moments
        _adamw("adamw32_model_f32", "f32", 32, False, 8, 640, 1999, False),
        # a half-billion-parameter model in bfloat16 with binary32 master weights, 8-bit moments
        _adamw("adamw8_model_bf16", "bf16", 8, True, 24, 1280, 32003, False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention_fwd", "attention_bwd", "attention_bwd", "qk_fwd", "qk_bwd", "adamw"])
    if op.startswith("attention"):
        kv = rng.choice([1, 2, 3, 4, 8])
        heads = kv * rng.choice([1, 2, 3, 4, 6])
        dim = rng.choice([32, 64, 64, 72, 96, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        causal = rng.random() < 0.6
        room = 8 * 16384 * 16384 // 4 // heads               # scores of one head in the plain form
        if rng.random() < 0.35:
            tokens, docs = _log_int(rng, 64, 12000), rng.randint(1, 24)
            case = _attn("", op, dtype, 1, tokens, tokens, heads, kv, dim, causal, False, docs)
            while docs * _longest(case) ** 2 > room:
                case["q_len"] = case["k_len"] = case["q_len"] * 4 // 5
        else:
            q_len = _log_int(rng, 1, min(9000, math.isqrt(room)))
            k_len = q_len if rng.random() < 0.7 else _log_int(rng, 1, min(9000, math.isqrt(room)))
            batch = rng.randint(1, max(1, min(16, room // (q_len * k_len))))
            case = _attn("", op, dtype, batch, q_len, k_len, heads, kv, dim, causal, q_len == k_len and rng.random() < 0.5)
    elif op.startswith("qk"):
        dim = rng.choice([32, 64, 80, 96, 128, 128, 256])
        rot = dim if rng.random() < 0.6 else dim // 2
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4, 7])
        tokens = _log_int(rng, 1, max(2, 4 * 8192 * 40 * 128 // ((heads + kv) * dim)))
        batch = rng.choice([1, 1, 2, 3])
        case = _qk("", op, rng.choice(["bf16", "bf16", "f16", "f32"]), batch, max(1, tokens // batch), heads, kv, dim,
                   rot, rng.random() < 0.3, rng.random() < 0.5)
    else:
        dtype = rng.choice(["f32", "bf16", "f16"])
        master = dtype != "f32" and rng.random() < 0.7
        bits = rng.choice([8, 8, 32])
        case = _adamw("", dtype, bits, master, rng.randint(1, 16), 8 * _log_int(rng, 2, 90), _log_int(rng, 100, 32000),
                      rng.random() < 0.5)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _shapes(case):
    """The tensors of a small transformer: per layer two norms, the projections and the biases; with `odd`, sizes
    that are no multiple of a block, a scalar among them."""
    w, shapes = case["width"], []
    for _ in range(case["layers"]):
        shapes += [(w,), (3 * w, w), (w, w), (w,), (4 * w, w), (4 * w,), (w, 4 * w)]
        if case["odd"]:
            shapes += [(w + 1, 7), (1,), (w - 3,)]
    if case["vocab"]:
        shapes.append((case["vocab"], w))
    return shapes


def _layout(case):
    """[(offset, elements, shape)] of the tensors in one buffer, each starting on a block; and the buffer's length."""
    at, out = 0, []
    for shape in _shapes(case):
        n = math.prod(shape)
        out.append((at, n, shape))
        at += -(-n // BLOCK) * BLOCK
    return out, at


def _doc_offsets(case):
    """Boundaries of the packed documents: unequal, fixed by the case (one of them may be empty)."""
    total, docs, at, cuts = case["q_len"], case["docs"], 0, []
    for i in range(docs - 1):
        at += int((total - at) * (0.15 + 0.6 * ((i * 7919 + total) % 101) / 101) * 2 / (docs - i + 1))
        cuts.append(at)
    return [0] + cuts + [total]


def _longest(case):
    cuts = _doc_offsets(case)
    return max(y - x for x, y in zip(cuts, cuts[1:]))


def _quantise(x, positive):
    """Codes and scales of an 8-bit moment (nearest rounding: these are a program's earlier state)."""
    rows = x.view(-1, BLOCK)
    top = rows.abs().amax(1)
    codes = (rows * (448.0 / top.clamp_min(1e-30))[:, None]).clamp(-448.0, 448.0)
    if positive:
        codes = torch.where(codes > 0, codes.clamp_min(2.0 ** -9), codes)
    return codes.to(torch.float8_e4m3fn).view(-1), top * (1.0 / 448.0)


def prepare(case, seed):
    dev, op, dtype = torch.device("cuda"), case["op"], DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device=dev) * std).to(to)

    s = {"case": case}
    if op.startswith("attention"):
        h, hk, d, b, lq, lk = (case[x] for x in ("heads", "kv_heads", "head_dim", "batch", "q_len", "k_len"))
        if case["fused"]:                                   # one projection's output: heads of q, k and v side by side
            qkv = normal(b, lq, h + 2 * hk, d)
            s["q"], s["k"], s["v"] = qkv[:, :, :h], qkv[:, :, h:h + hk], qkv[:, :, h + hk:]
        else:
            s["q"], s["k"], s["v"] = normal(b, lq, h, d), normal(b, lk, hk, d), normal(b, lk, hk, d)
        s["kw"] = {"causal": case["causal"]}
        if case["docs"]:
            cuts = _doc_offsets(case)
            s["q"], s["k"], s["v"] = s["q"][0], s["k"][0], s["v"][0]
            s["offsets"] = torch.tensor(cuts, dtype=torch.int32, device=dev)
            longest = _longest(case)
            s["kw"] |= {"q_offsets": s["offsets"], "k_offsets": s["offsets"], "max_q_len": longest, "max_k_len": longest}
        if op == "attention_bwd":
            s["out"], s["lse"] = _plain_attention_fwd(s)    # what the forward pass of the step left behind
            s["grad_out"] = normal(*s["out"].shape)
    elif op.startswith("qk"):
        b, n, h, hk, d, r = (case[x] for x in ("batch", "length", "heads", "kv_heads", "head_dim", "rotary_dim"))
        qkv = normal(b, n, h + 2 * hk, d, std=1.5)
        s["q"], s["k"] = qkv[:, :, :h], qkv[:, :, h:h + hk]
        s["q_weight"], s["k_weight"] = 1 + normal(d, std=0.2, to=torch.float32), 1 + normal(d, std=0.2, to=torch.float32)
        rows = n + 100 if case["positions"] else n
        freq = 10000.0 ** (-torch.arange(0, r, 2, device=dev, dtype=torch.float32) / r)
        angle = torch.arange(rows, device=dev, dtype=torch.float32)[:, None] * freq
        s["cos"], s["sin"] = angle.cos(), angle.sin()
        s["kw"] = {"eps": 1e-6, "interleaved": case["interleaved"], "positions": None}
        if case["positions"]:
            s["kw"]["positions"] = torch.randint(0, rows, (b, n), generator=gen, device=dev, dtype=torch.int32)
        if op == "qk_bwd":
            s["grad_q"], s["grad_k"] = normal(b, n, h, d), normal(b, n, hk, d)
    else:
        layout, total = _layout(case)
        keep = torch.zeros(total, device=dev, dtype=torch.bool)             # the elements between two tensors stay zero
        for at, n, _ in layout:
            keep[at:at + n] = True
        s["size"], s["layout"] = total, layout
        value = normal(total, std=0.02, to=torch.float32) * keep
        m = normal(total, std=1e-3, to=torch.float32) * keep
        r = (normal(total, std=1e-3, to=torch.float32).abs() + 1e-3) * keep  # the root of the second moment
        s["param"] = value.to(dtype)
        s["master"] = value if case["master"] else None
        s["grad"] = normal(total, std=2e-3) * keep
        if case["state_bits"] == 8:
            (s["m"], s["m_scale"]), (s["v"], s["v_scale"]) = _quantise(m, False), _quantise(r, True)
        else:
            s["m"], s["v"], s["m_scale"], s["v_scale"] = m, r * r, None, None
        del keep, value, m, r
        s["kw"] = {"step": 1000, "lr": 1e-3, "betas": (0.9, 0.999), "eps": 1e-8, "weight_decay": 0.1, "seed": seed & 0xFFFFFFFF}
        if own:                                             # the handle that an optimizer keeps
            import paper_2202_00441_b200 as fb

            def cut(flat):
                return None if flat is None else [flat[at:at + n].view(shape) for at, n, shape in layout]

            def cut_scales(flat):
                return None if flat is None else [flat[at // BLOCK:at // BLOCK + -(-n // BLOCK)] for at, n, _ in layout]

            s["tensors"] = fb.fewbit_adamw_create(cut(s["param"]), cut(s["m"]), cut(s["v"]), cut_scales(s["m_scale"]),
                                                  cut_scales(s["v_scale"]), cut(s["master"]))
            s["grads"] = cut(s["grad"])
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------

def _pad_index(offsets, longest):
    """(row of every padded place, whether it is one) for sequences packed at `offsets`."""
    at = torch.arange(longest, device=offsets.device)
    first, n = offsets[:-1].long(), (offsets[1:] - offsets[:-1]).long()
    valid = at[None, :] < n[:, None]
    return torch.where(valid, first[:, None] + at, 0), valid


def _unpad(padded, offsets, rows):
    t = torch.arange(rows, device=padded.device)
    seq = (t[:, None] >= offsets[None, 1:]).sum(1)
    return padded[seq, t - offsets[seq].long()]


def _plain_scores(s):
    """32-bit q, k, v as (batch, kv_heads, group, length, dim) and the masked scores."""
    q, k, v, kw = s["q"], s["k"], s["v"], s["kw"]
    d = q.shape[-1]
    if "offsets" in s:
        qi, q_valid = _pad_index(kw["q_offsets"], kw["max_q_len"])
        ki, k_valid = _pad_index(kw["k_offsets"], kw["max_k_len"])
        q, k, v = q[qi], k[ki], v[ki]
    b, lq, h, _ = q.shape
    lk, hk = k.shape[1], k.shape[2]
    qf = q.float().transpose(1, 2).reshape(b, hk, h // hk, lq, d)
    kf, vf = (x.float().transpose(1, 2).unsqueeze(2) for x in (k, v))
    scores = torch.matmul(qf, kf.transpose(-1, -2)) * d ** -0.5
    if "offsets" in s:
        shift = (kw["k_offsets"].diff() - kw["q_offsets"].diff())[:, None, None].long()
        seen = k_valid[:, None, :] & q_valid[:, :, None]
    else:
        shift, seen = lk - lq, None
    if kw["causal"]:
        below = torch.arange(lk, device=q.device)[None, :] <= torch.arange(lq, device=q.device)[:, None] + shift
        seen = below if seen is None else seen & below
    if seen is not None:
        if seen.dim() == 3:
            seen = seen[:, None, None]
        scores = scores.masked_fill(~seen, -math.inf)
    return qf, kf, vf, scores


def _plain_softmax(scores):
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (scores - top).exp()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)                   # -inf for a row that sees nothing
    return p / torch.where(total == 0, 1.0, total), lse


def _heads_last(x, s, name):
    """(batch, kv_heads, group, length, dim) in 32 bits -> the layout and type of s[name]."""
    x = x.flatten(1, 2).transpose(1, 2)
    if "offsets" in s:
        x = _unpad(x, s["offsets"], s[name].shape[0])
    return x.to(s[name].dtype).contiguous()


def _plain_attention_fwd(s):
    _, _, vf, scores = _plain_scores(s)
    p, lse = _plain_softmax(scores)
    out = torch.matmul(p, vf)
    lse = lse.flatten(1, 2)
    if "offsets" in s:
        lse = _unpad(lse.transpose(1, 2), s["offsets"], s["q"].shape[0]).T.contiguous()
    return _heads_last(out, s, "q"), lse


def _plain_attention_bwd(s):
    qf, kf, vf, scores = _plain_scores(s)
    g = s["grad_out"]
    if "offsets" in s:
        gi, valid = _pad_index(s["kw"]["q_offsets"], s["kw"]["max_q_len"])
        g = g[gi] * valid[:, :, None, None]
    gf = g.float().transpose(1, 2).reshape(qf.shape)
    p, _ = _plain_softmax(scores)
    del scores
    dv = torch.matmul(p.transpose(-1, -2), gf).sum(2, keepdim=True)
    dp = torch.matmul(gf, vf.transpose(-1, -2))
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * qf.shape[-1] ** -0.5
    del p, dp
    dq = torch.matmul(ds, kf)
    dk = torch.matmul(ds.transpose(-1, -2), qf).sum(2, keepdim=True)
    return _heads_last(dq, s, "q"), _heads_last(dk, s, "k"), _heads_last(dv, s, "v")


def _plain_rotation(s):
    """cos and sin of every token's pairs, with a dimension for the heads."""
    b, n = s["q"].shape[:2]
    at = s["kw"]["positions"]
    at = torch.arange(n, device=s["q"].device).expand(b, n) if at is None else at.long()
    return s["cos"][at].unsqueeze(2), s["sin"][at].unsqueeze(2)


def _pairs(x, r, interleaved):
    return (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])


def _rotate(x, cos, sin, interleaved):
    r = 2 * cos.shape[-1]
    a, b = _pairs(x, r, interleaved)
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, v], -1).flatten(-2) if interleaved else torch.cat([u, v], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_qk_fwd(s):
    cos, sin = _plain_rotation(s)

    def one(x, w):
        f = x.float()
        f = f * (f.square().mean(-1, keepdim=True) + s["kw"]["eps"]).rsqrt() * w
        return _rotate(f, cos, sin, s["kw"]["interleaved"]).to(x.dtype)

    return one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])


def _plain_qk_bwd(s):
    cos, sin = _plain_rotation(s)

    def one(g, x, w):
        f = x.float()
        rstd = (f.square().mean(-1, keepdim=True) + s["kw"]["eps"]).rsqrt()
        unit = f * rstd
        g = _rotate(g.float(), cos, -sin, s["kw"]["interleaved"])
        dw = (g * unit).sum((0, 1, 2))
        g = g * w
        dx = rstd * (g - unit * (g * unit).mean(-1, keepdim=True))
        return dx.to(x.dtype), dw

    dq, dqw = one(s["grad_q"], s["q"], s["q_weight"])
    dk, dkw = one(s["grad_k"], s["k"], s["k_weight"])
    return dq, dk, dqw, dkw


def _random_bits(n, seed, device):
    """32 random bits for every element: the generator's counter is the element's place."""
    x = (torch.arange(n, device=device) * 0x9E3779B1 + seed) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x6A09E667) & 0xFFFFFFFF
    x = ((x ^ (x >> 13)) * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _stochastic_float8(x, noise, positive):
    """Blocks scaled to 448 and rounded up with the probability of what is cut off (`noise`: 20 random bits)."""
    rows = x.view(-1, BLOCK)
    top = rows.abs().amax(1)
    u = (rows.abs() * torch.where(top > 0, 448.0 / top, 0.0)[:, None]).view(-1)
    small = u < 2.0 ** -6                                   # float8's subnormals: one fixed step
    bits = torch.where(small, u + 2.0 ** -6, u).view(torch.int32) + noise.int()
    code = torch.minimum((bits >> 20) - torch.where(small, 968, 960), torch.full((), 126, device=x.device, dtype=torch.int32))
    if positive:
        code = torch.where(u > 0, code.clamp_min(1), code)
    code = torch.where(x < 0, code + 128, code).to(torch.uint8)
    return code.view(torch.float8_e4m3fn), top * (1.0 / 448.0)


def _plain_adamw(s):
    kw, eight = s["kw"], s["m_scale"] is not None
    b1, b2 = kw["betas"]
    g = s["grad"].float()
    if eight:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    p = s["param"].float() if s["master"] is None else s["master"]
    bc1, bc2 = 1 - b1 ** kw["step"], 1 - b2 ** kw["step"]
    p = p * (1 - kw["lr"] * kw["weight_decay"]) - (kw["lr"] / bc1) * (m / (v.sqrt() * bc2 ** -0.5 + kw["eps"]))
    if s["master"] is not None:
        s["master"].copy_(p)
    s["param"].copy_(p)
    if eight:
        noise = _random_bits(s["size"], kw["seed"], p.device)
        for name, x, cut, positive in (("m", m, (noise & 0xFFFF) << 4, False), ("v", v.sqrt(), (noise >> 16) << 4, True)):
            codes, scale = _stochastic_float8(x, cut, positive)
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def _adamw_outputs(s):
    # the 8-bit moments are float8 tensors: they come back as such, with their scales
    return {k: s[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale")}


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "attention_fwd":
            return _plain_attention_fwd(s)
        if op == "attention_bwd":
            return _plain_attention_bwd(s)
        if op == "qk_fwd":
            return _plain_qk_fwd(s)
        if op == "qk_bwd":
            return _plain_qk_bwd(s)
        _plain_adamw(s)
        return _adamw_outputs(s)

    import paper_2202_00441_b200 as fb

    if op == "attention_fwd":
        return fb.fewbit_attention_fwd(s["q"], s["k"], s["v"], **s["kw"])
    if op == "attention_bwd":
        return fb.fewbit_attention_bwd(s["grad_out"], s["q"], s["k"], s["v"], s["out"], s["lse"], **s["kw"])
    if op == "qk_fwd":
        return fb.fewbit_qk_norm_rope_fwd(s["q"], s["k"], s["q_weight"], s["k_weight"], s["cos"], s["sin"], **s["kw"])
    if op == "qk_bwd":
        return fb.fewbit_qk_norm_rope_bwd(s["grad_q"], s["grad_k"], s["q"], s["k"], s["q_weight"], s["k_weight"],
                                          s["cos"], s["sin"], **s["kw"])
    fb.fewbit_adamw_step(s["tensors"], s["grads"], **s["kw"])
    return _adamw_outputs(s)


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def _seen_pairs(case):
    """(query, key) pairs that the mask leaves, over all sequences of the batch."""
    if case["docs"]:
        cuts = _doc_offsets(case)
        spans = [(y - x, y - x) for x, y in zip(cuts, cuts[1:])]
    else:
        spans = [(case["q_len"], case["k_len"])] * case["batch"]
    total = 0
    for lq, lk in spans:
        if case["causal"]:                                   # row i sees max(0, i + 1 + lk - lq) keys
            first = max(0, lq - lk)
            rows, low = lq - first, max(1, 1 + lk - lq)
            total += rows * low + rows * (rows - 1) // 2 if rows else 0
        else:
            total += lq * lk
    return total


def work(case):
    op, e = case["op"], BYTES[case["dtype"]]
    if op.startswith("attention"):
        q = case["batch"] * case["q_len"] * case["heads"] * case["head_dim"] * e
        k = case["batch"] * case["k_len"] * case["kv_heads"] * case["head_dim"] * e
        rows = case["batch"] * case["q_len"] * case["heads"] * 4
        pair = 2 * _seen_pairs(case) * case["heads"] * case["head_dim"]
        if op == "attention_fwd":                            # q, k, v in; out and lse out; two products
            return {"bytes": 2 * q + 2 * k + rows, "flops": 2 * pair}
        return {"bytes": 4 * q + 4 * k + rows, "flops": 5 * pair}   # five products; the scores are recomputed
    if op.startswith("qk"):
        tokens = case["batch"] * case["length"]
        x = tokens * (case["heads"] + case["kv_heads"]) * case["head_dim"]
        table = min(tokens, case["length"] + 100) * case["rotary_dim"] * 4
        return {"bytes": (2 if op == "qk_fwd" else 3) * x * e + table, "flops": (6 if op == "qk_fwd" else 14) * x}
    n = sum(math.prod(shape) for shape in _shapes(case))
    moments = 4 * (1 + 4 / BLOCK) if case["state_bits"] == 8 else 16
    weights = e + 8 if case["master"] else 2 * e             # a master copy is read and written, the parameter only written
    return {"bytes": n * (e + weights + moments), "flops": 20 * n}


def _exact_attention(s, case):
    dev = s["q"].device
    packed = "offsets" in s
    cuts = s["offsets"].tolist() if packed else None
    backward = case["op"] == "attention_bwd"
    names = ("q", "k", "v") + (("grad_out",) if backward else ())
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    spans = list(zip(cuts, cuts[1:])) if packed else range(case["batch"])
    lead = s["q"].shape[:-2]
    if backward:
        out = [torch.zeros(s[n].shape, dtype=torch.float64, device=dev) for n in ("q", "k", "v")]
    else:
        out = [torch.zeros(s["q"].shape, dtype=torch.float64, device=dev),
               torch.zeros((h, *lead) if packed else (lead[0], h, lead[1]), dtype=torch.float64, device=dev)]
    for span in spans:
        rows = slice(*span) if packed else span
        for i in range(h):
            x = {n: s[n][rows][:, i // (h // hk) if n in "kv" else i].double() for n in names}
            lq, lk = x["q"].shape[0], x["k"].shape[0]
            if not lq or not lk:
                if not backward and lq:
                    (out[1][i, rows] if packed else out[1][rows, i]).fill_(-math.inf)
                continue
            z = x["q"] @ x["k"].T / math.sqrt(d)
            if case["causal"]:
                z.masked_fill_(torch.ones(lq, lk, dtype=torch.bool, device=dev).triu(1 + lk - lq), -math.inf)
            lse = torch.logsumexp(z, 1)
            p = z.sub_(lse[:, None]).exp_().nan_to_num_(nan=0.0)
            if not backward:
                out[0][rows][:, i] = p @ x["v"]
                if packed:
                    out[1][i, rows] = lse
                else:
                    out[1][rows, i] = lse
                continue
            g = x["grad_out"]
            out[2][rows][:, i // (h // hk)] += p.T @ g
            dz = g @ x["v"].T
            dz.sub_((p * dz).sum(1, keepdim=True)).mul_(p).div_(math.sqrt(d))
            out[0][rows][:, i] = dz @ x["k"]
            out[1][rows][:, i // (h // hk)] += dz.T @ x["q"]
            del z, p, dz
    return tuple(out)


def _exact_qk(s, case):
    b, n, r = case["batch"], case["length"], case["rotary_dim"]
    dev = s["q"].device
    at = s["kw"]["positions"]
    at = torch.arange(n, device=dev).repeat(b, 1) if at is None else at.long()
    turn = torch.complex(s["cos"].double(), s["sin"].double())[at][:, :, None]
    order = torch.arange(r, device=dev)
    order = order.view(-1, 2) if case["interleaved"] else order.view(2, -1).T       # the two places of each pair

    def rotate(x, by):
        z = torch.complex(x[..., order[:, 0]], x[..., order[:, 1]]) * by
        y = x.clone()
        y[..., order[:, 0]], y[..., order[:, 1]] = z.real, z.imag
        return y

    outs, sums = [], []
    for x, w, g in ((s["q"], s["q_weight"], s.get("grad_q")), (s["k"], s["k_weight"], s.get("grad_k"))):
        x, w = x.double(), w.double()
        norm = torch.sqrt(x.pow(2).mean(-1, keepdim=True) + s["kw"]["eps"])
        if g is None:
            outs.append(rotate(x / norm * w, turn))
            continue
        g = rotate(g.double(), turn.conj())
        sums.append((g * x / norm).flatten(0, 2).sum(0))
        g = g * w
        outs.append(g / norm - x * (g * x).mean(-1, keepdim=True) / norm ** 3)
    return tuple(outs + sums)


def _exact_round(u, chance, positive):
    """|u| <= 448 to a neighbouring float8 value, up where `chance` (in [0, 1)) passes the distance to the upper one."""
    step = torch.exp2(torch.floor(torch.log2(u.clamp_min(2.0 ** -6))) - 3)
    q = torch.floor(u / step + chance) * step
    if positive:
        q = torch.where((u > 0) & (q == 0), 2.0 ** -9, q)
    return q.clamp_max(448.0)


def _exact_adamw(s, case):
    kw, eight = s["kw"], case["state_bits"] == 8
    b1, b2 = kw["betas"]
    n, t = s["size"], kw["step"]
    out = {k: None for k in ("param", "master", "m", "v", "m_scale", "v_scale")}
    wide = [torch.empty(n, dtype=torch.float64, device=s["param"].device) for _ in range(3)]
    scales = [torch.empty(n // BLOCK, dtype=torch.float64, device=s["param"].device) for _ in range(2)]
    piece = 1 << 25
    for at in range(0, n, piece):
        i = slice(at, min(n, at + piece))
        ib = slice(i.start // BLOCK, i.stop // BLOCK)
        g = s["grad"][i].double()
        m, v = s["m"][i].double(), s["v"][i].double()
        if eight:
            m = (m.view(-1, BLOCK) * s["m_scale"][ib].double()[:, None]).view(-1)
            v = (v.view(-1, BLOCK) * s["v_scale"][ib].double()[:, None]).view(-1) ** 2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
        p = (s["master"] if s["master"] is not None else s["param"])[i].double()
        p = p - kw["lr"] * kw["weight_decay"] * p - kw["lr"] * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + kw["eps"])
        wide[0][i] = p
        if not eight:
            wide[1][i], wide[2][i] = m, v
            continue
        bits = torch.arange(i.start, i.stop, device=p.device)
        bits = (bits * 0x9E3779B1 + kw["seed"]) % 2 ** 32
        bits = ((bits ^ bits // 2 ** 15) * 0x6A09E667) % 2 ** 32
        bits = ((bits ^ bits // 2 ** 13) * 0xBB67AE85) % 2 ** 32
        bits = bits ^ bits // 2 ** 16
        for k, x, half in ((0, m, bits % 2 ** 16), (1, v.sqrt(), bits // 2 ** 16)):
            top = x.abs().view(-1, BLOCK).amax(1)
            scales[k][ib] = top / 448
            u = x.abs().view(-1, BLOCK) * torch.where(top > 0, 448 / top, 0.0)[:, None]
            q = _exact_round(u.view(-1), half.double() / 2 ** 16, k == 1)
            wide[1 + k][i] = torch.where(x < 0, -q, q)
    out["param"], out["m"], out["v"] = wide
    if case["master"]:
        out["master"] = wide[0]
    if eight:
        out["m_scale"], out["v_scale"] = scales
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("attention"):
        if 10 * _seen_pairs(case | {"causal": False}) * case["heads"] * case["head_dim"] > 1e14:
            return None
        return _exact_attention(s, case)
    if case["op"].startswith("qk"):
        return _exact_qk(s, case)
    return _exact_adamw(s, case)
