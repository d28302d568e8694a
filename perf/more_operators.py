"""What the operators of a transformer block around attention's scores and the residual stream are measured on.

Four families, each with its plain form (elementary torch operations in 32 bits) and the library's kernels:

* attention, forward and backward, whose scores are capped by a tanh, biased by the distance of key and row, and masked by
  documents and a prefix;
* the same with a learned bias of relative positions by buckets: the table is spread over the distances, and its gradient
  comes back from the scores';
* dropout whose mask is drawn again in the backward pass, never stored, with the residual's addition;
* the RMS norm of the residual stream after a branch has been added to it (through dropout), its result in the tensors' type
  or in 8 bits with a scale for each row, forward and backward.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
FLOAT8_MAX = 448.0
PHILOX_MULTIPLIERS = (0xD2511F53, 0xCD9E8D57)       # Salmon, Moraes, Dror and Shaw, Parallel random numbers: as easy as 1, 2, 3 (2011)
PHILOX_KEYS = (0x9E3779B9, 0xBB67AE85)


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def _attn(name, op, dtype, batch, q_len, k_len, heads, kv_heads, head_dim, causal, cap=0.0, slopes=False, prefix=0, docs=0,
          buckets=0, max_distance=0, both=False, table="f32"):
    """prefix: the longest of the batch's prefixes; docs: documents in each sequence; buckets: of the learned bias."""
    return {"name": name, "op": op, "dtype": dtype, "batch": batch, "q_len": q_len, "k_len": k_len, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "cap": cap, "slopes": slopes, "prefix": prefix,
            "docs": docs, "buckets": buckets, "max_distance": max_distance, "both": both, "table": table}


def _drop(name, op, dtype, rows, width, p, residual):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "width": width, "p": p, "residual": residual}


def _norm(name, op, dtype, rows, width, p, bits):
    """bits: 0 for a result in the tensors' type, 8 for float8 codes with a scale for each row."""
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "width": width, "p": p, "bits": bits}


def listed():
    return [
        # a short prompt through a model with capped scores: latency
        _attn("score_fwd_short_f16", "attention_fwd", "f16", 2, 77, 77, 4, 4, 64, True, cap=30.0),
        # long-context pre-training, a row of 16384 tokens packed from a dozen documents, capped scores
        _attn("score_fwd_docs_bf16", "attention_fwd", "bf16", 1, 16384, 16384, 8, 2, 128, True, cap=50.0, docs=12),
        # fine-tuning with a prefix that sees itself in both directions and a linear bias by distance, odd lengths
        _attn("score_bwd_prefix_f16", "attention_bwd", "f16", 3, 1111, 1111, 6, 2, 64, True, slopes=True, prefix=400),
        # a pre-training micro-batch with capped scores
        _attn("score_bwd_train_bf16", "attention_bwd", "bf16", 4, 2048, 2048, 16, 4, 128, True, cap=50.0),
        # a decoder's rows over an encoder's odd number of keys, learned bias of one direction
        _attn("bias_fwd_odd_f16", "attention_fwd", "f16", 2, 333, 517, 8, 8, 64, True, buckets=32, max_distance=128),
        # an encoder's training micro-batch, learned bias of both directions
        _attn("bias_bwd_encoder_bf16", "attention_bwd", "bf16", 8, 1024, 1024, 12, 12, 64, False, buckets=32, max_distance=128, both=True),
        # an adapter's few activations in binary32: latency
        _drop("drop_bwd_few_f32", "dropout_bwd", "f32", 7, 333, 0.1, False),
        # a training micro-batch's branch, dropped and added to the residual stream
        _drop("drop_fwd_train_bf16", "dropout_fwd", "bf16", 16384, 4096, 0.1, True),
        # a handful of tokens in binary32: latency
        _norm("norm_bwd_few_f32", "norm_bwd", "f32", 5, 640, 0.0, 0),
        # an odd batch whose next product takes 8 bits
        _norm("norm_fwd_8bit_f16", "norm_fwd", "f16", 2999, 1288, 0.0, 8),
        # a training micro-batch with dropout of the branch
        _norm("norm_fwd_train_bf16", "norm_fwd", "bf16", 16384, 4096, 0.1, 0),
        # and its backward pass
        _norm("norm_bwd_train_bf16", "norm_bwd", "bf16", 16384, 4096, 0.1, 0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention_fwd", "attention_fwd", "attention_bwd", "attention_bwd", "dropout_fwd", "dropout_bwd", "norm_fwd", "norm_bwd"])
    if op.startswith("attention"):
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 3, 4])
        dim = rng.choice([32, 64, 64, 72, 96, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "f16"])
        room = 16384 * 16384 // 4 // heads                       # scores of one head in the plain form
        q_len = _log_int(rng, 1, min(6000, math.isqrt(room)))
        k_len = q_len if rng.random() < 0.7 else _log_int(rng, 1, min(6000, math.isqrt(room)))
        batch = rng.randint(1, max(1, min(8, room // (q_len * k_len))))
        case = _attn("", op, dtype, batch, q_len, k_len, heads, kv, dim, rng.random() < 0.6)
        kind = rng.choice(["cap", "cap", "slopes", "table", "table", "none"])
        if kind == "cap":
            case["cap"] = rng.choice([5.0, 20.0, 30.0, 50.0])
        elif kind == "slopes":
            case["slopes"] = True
        elif kind == "table":
            case["both"] = not case["causal"]
            case["buckets"], case["max_distance"] = rng.choice([(32, 128), (32, 128), (16, 64), (64, 300)])
            case["table"] = rng.choice(["f32", dtype])
        if case["causal"] and (kind == "none" or rng.random() < 0.4):
            case["prefix"] = _log_int(rng, 1, k_len)
        if not case["prefix"] and (kind == "none" or rng.random() < 0.4):
            case["docs"] = rng.randint(2, 12)
    elif op.startswith("dropout"):
        width = _log_int(rng, 8, 8192)
        rows = _log_int(rng, 1, 16384 * 4096 // width)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        case = _drop("", op, dtype, max(1, rows // (BYTES[dtype] // 2)), width, rng.choice([0.05, 0.1, 0.25, 0.5]),
                     op == "dropout_fwd" and rng.random() < 0.6)
    else:
        width = 8 * _log_int(rng, 4, 1024) if rng.random() < 0.8 else _log_int(rng, 32, 8192)
        rows = _log_int(rng, 1, 16384 * 4096 // width)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        case = _norm("", op, dtype, max(1, rows // (BYTES[dtype] // 2)), width, rng.choice([0.0, 0.1, 0.3]),
                     8 if op == "norm_fwd" and rng.random() < 0.4 else 0)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _cuts(case, b):
    """Boundaries of the documents of sequence b: unequal, fixed by the case."""
    total, docs, at, cuts = case["q_len"], case["docs"], 0, []
    for i in range(docs - 1):
        at += int((total - at) * (0.15 + 0.6 * ((i * 7919 + total + 31 * b) % 101) / 101) * 2 / (docs - i + 1))
        cuts.append(at)
    return [0] + cuts + [total]


def _key_cuts(case, b):
    """The same boundaries on the keys' axis."""
    return [x * case["k_len"] // case["q_len"] for x in _cuts(case, b)]


def _prefixes(case):
    return [max(1, case["prefix"] * (case["batch"] - b) // case["batch"]) for b in range(case["batch"])]


def prepare(case, seed):
    dev, op, dtype = torch.device("cuda"), case["op"], DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape, std=1.0, to=dtype):
        return (torch.randn(*shape, generator=gen, device=dev) * std).to(to)

    s = {"case": case}
    if op.startswith("attention"):
        h, hk, d, b, lq, lk = (case[x] for x in ("heads", "kv_heads", "head_dim", "batch", "q_len", "k_len"))
        size = 3.0 if case["cap"] else 1.0                       # capped scores are large ones
        s["q"], s["k"], s["v"] = normal(b, lq, h, d, std=size), normal(b, lk, hk, d), normal(b, lk, hk, d)
        s["kw"] = {"causal": case["causal"]}
        if case["cap"]:
            s["kw"]["cap"] = case["cap"]
        if case["slopes"]:                                       # a geometric sequence over the heads
            s["kw"]["slopes"] = torch.exp2(-8.0 * torch.arange(1, h + 1, device=dev, dtype=torch.float32) / h)
        if case["prefix"]:
            s["kw"]["prefix_lens"] = torch.tensor(_prefixes(case), dtype=torch.int32, device=dev)
        if case["docs"]:
            for name, cuts, n in (("q_documents", _cuts, lq), ("k_documents", _key_cuts, lk)):
                rows = []
                for i in range(b):
                    lengths = torch.tensor(cuts(case, i)).diff()
                    rows.append(torch.repeat_interleave(torch.arange(len(lengths)), lengths))
                s["kw"][name] = torch.stack(rows).to(dev, torch.int32)
        if case["buckets"]:
            s["table"] = normal(case["buckets"], h, std=0.7, to=DTYPES[case["table"]])
        if op == "attention_bwd":
            s["out"], s["lse"] = _plain_attention_fwd(s)         # what the forward pass of the step left behind
            s["grad_out"] = normal(*s["out"].shape)
    elif op.startswith("dropout"):
        n, w = case["rows"], case["width"]
        s["x"] = normal(n, w)
        s["residual"] = normal(n, w, std=2.0) if case["residual"] else None
        s["kw"] = {"p": case["p"], "seed": (seed * 0x9E3779B97F4A7C15 + 1) & 0x7FFFFFFFFFFFFFFF, "place": 3}
    else:
        n, w = case["rows"], case["width"]
        s["weight"] = 1 + normal(w, std=0.2, to=torch.float32)
        s["kw"] = {"eps": EPS, "p": case["p"], "seed": (seed * 0x9E3779B97F4A7C15 + 1) & 0x7FFFFFFFFFFFFFFF, "place": 5}
        if op == "norm_fwd":
            s["x"], s["residual"] = normal(n, w), normal(n, w, std=2.0)
        else:
            s["h"], s["grad_y"], s["grad_h"] = normal(n, w, std=2.0), normal(n, w), normal(n, w, std=0.5)
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------

def _bucket_of(distance, buckets, most, both):
    """The bucket of each distance (key's place minus row's): exact up to half the buckets of a direction, then logarithmic."""
    n = buckets // 2 if both else buckets
    far = distance.abs() if both else (-distance).clamp_min(0)
    exact = n // 2
    # in 64 bits; a distance whose logarithm falls on a border by the formula belongs above it
    large = exact + ((far.clamp_min(1).double() / exact).log() / math.log(most / exact) * (n - exact) + 1e-9).floor().long()
    bucket = torch.where(far < exact, far, large.clamp_max(n - 1))
    return torch.where(distance > 0, bucket + n, bucket) if both else bucket


def _distances(s):
    """(q_len, k_len): how far each key lies behind (negative) or ahead of each row, the last row and key level."""
    lq, lk, dev = s["q"].shape[1], s["k"].shape[1], s["q"].device
    return torch.arange(lk, device=dev)[None, :] - torch.arange(lq, device=dev)[:, None] - (lk - lq)


def _plain_spread(s):
    """(heads, 2 R + 1): the learned bias of every distance from -R to R."""
    case, most = s["case"], s["case"]["max_distance"]
    at = torch.arange(-most, most + 1, device=s["q"].device)
    return s["table"].float()[_bucket_of(at, case["buckets"], most, case["both"])].T.contiguous()


def _plain_scores(s):
    """32-bit q, k, v as (batch, kv_heads, group, length, dim), the scores with bias and mask, and the tanh of capped ones."""
    q, k, v, kw, case = s["q"], s["k"], s["v"], s["kw"], s["case"]
    b, lq, h, d = q.shape
    lk, hk = k.shape[1], k.shape[2]
    qf = q.float().transpose(1, 2).reshape(b, hk, h // hk, lq, d)
    kf, vf = (x.float().transpose(1, 2).unsqueeze(2) for x in (k, v))
    scores = torch.matmul(qf, kf.transpose(-1, -2)) * d ** -0.5
    bent = None
    if "cap" in kw:
        bent = torch.tanh(scores / kw["cap"])
        scores = bent * kw["cap"]
    away = _distances(s)
    if "slopes" in kw:
        scores = scores - kw["slopes"].view(hk, -1, 1, 1) * away.abs()
    if "table" in s:
        most = case["max_distance"]
        scores = scores + _plain_spread(s)[:, away.clamp(-most, most) + most].view(hk, -1, lq, lk)
    seen = None
    if kw["causal"]:
        seen = (away <= 0)[None]
        if "prefix_lens" in kw:
            seen = seen | (torch.arange(lk, device=q.device) < kw["prefix_lens"][:, None])[:, None, :]
    if "q_documents" in kw:
        same = kw["q_documents"][:, :, None] == kw["k_documents"][:, None, :]
        seen = same if seen is None else seen & same
    if seen is not None:
        scores = scores.masked_fill(~seen[:, None, None], -math.inf)
    return qf, kf, vf, scores, bent


def _plain_softmax(scores):
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = (scores - top).exp()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)                        # -inf for a row that sees nothing
    return p / torch.where(total == 0, 1.0, total), lse


def _heads_last(x, like):
    """(batch, kv_heads, group, length, dim) in 32 bits -> the layout and type of `like`."""
    return x.flatten(1, 2).transpose(1, 2).to(like.dtype).contiguous()


def _plain_attention_fwd(s):
    _, _, vf, scores, _ = _plain_scores(s)
    p, lse = _plain_softmax(scores)
    return _heads_last(torch.matmul(p, vf), s["q"]), lse.flatten(1, 2)


def _sums_by_distance(ds, shift, most):
    """(heads, q_len, k_len) -> (heads, 2 R + 1): sums over the diagonals, what lies further than R at the ends."""
    h, lq, lk = ds.shape
    pad = torch.nn.functional.pad(ds, (lq, 0)).flatten(1)        # rows of lq + lk: each one's start moves by one place
    pad = torch.nn.functional.pad(pad, (0, lq)).view(h, lq, lq + lk + 1)
    diagonals = pad.sum(1, dtype=torch.float64)                  # place c holds key - row = c - lq
    to = (torch.arange(lq + lk + 1, device=ds.device) - lq - shift).clamp(-most, most) + most
    return torch.zeros(h, 2 * most + 1, dtype=torch.float64, device=ds.device).index_add_(1, to, diagonals)


def _plain_attention_bwd(s):
    qf, kf, vf, scores, bent = _plain_scores(s)
    case = s["case"]
    gf = s["grad_out"].float().transpose(1, 2).reshape(qf.shape)
    p, _ = _plain_softmax(scores)
    del scores
    dv = torch.matmul(p.transpose(-1, -2), gf).sum(2, keepdim=True)
    dp = torch.matmul(gf, vf.transpose(-1, -2))
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    del p, dp
    table = []
    if "table" in s:
        most = case["max_distance"]
        by_distance = _sums_by_distance(ds.flatten(1, 2).sum(0), case["k_len"] - case["q_len"], most)
        at = torch.arange(-most, most + 1, device=ds.device)
        bucket = _bucket_of(at, case["buckets"], most, case["both"])
        grad = torch.zeros(case["buckets"], case["heads"], dtype=torch.float64, device=ds.device).index_add_(0, bucket, by_distance.T)
        table = [grad.to(s["table"].dtype)]
    if bent is not None:
        ds = ds * (1 - bent * bent)
        del bent
    ds = ds * qf.shape[-1] ** -0.5
    dq = torch.matmul(ds, kf)
    dk = torch.matmul(ds.transpose(-1, -2), qf).sum(2, keepdim=True)
    return (_heads_last(dq, s["q"]), _heads_last(dk, s["k"]), _heads_last(dv, s["v"]), *table)


def _product(a, b):
    """High and low 32 bits of a * b for 32-bit values held in 64."""
    low = (a & 0xFFFF) * b
    high = (a >> 16) * b
    whole = (low >> 16) + high                                   # of at most 48 bits
    return whole >> 16, ((whole & 0xFFFF) << 16) | (low & 0xFFFF)


def _random_words(n, seed, place, device):
    """n words of 32 random bits: four for each count of the generator."""
    group = torch.arange((n + 3) // 4, device=device)
    c = [group & 0xFFFFFFFF, group >> 32, torch.full_like(group, place), torch.zeros_like(group)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        h0, l0 = _product(c[0], PHILOX_MULTIPLIERS[0])
        h1, l1 = _product(c[2], PHILOX_MULTIPLIERS[1])
        c = [h1 ^ c[1] ^ k[0], l1, h0 ^ c[3] ^ k[1], l0]
        k = [(k[0] + PHILOX_KEYS[0]) & 0xFFFFFFFF, (k[1] + PHILOX_KEYS[1]) & 0xFFFFFFFF]
    return torch.stack(c, 1).flatten()[:n]


def _plain_drop(x, kw):
    """x in 32 bits, dropped."""
    if not kw["p"]:
        return x
    kept = _random_words(x.numel(), kw["seed"], kw["place"], x.device) >= round(kw["p"] * 2 ** 32)
    return torch.where(kept.view(x.shape), x * (1 / (1 - kw["p"])), 0.0)


def _plain_dropout_fwd(s):
    y = _plain_drop(s["x"].float(), s["kw"])
    if s["residual"] is not None:
        y = s["residual"].float() + y
    return y.to(s["x"].dtype)


def _plain_norm_fwd(s):
    h = s["residual"].float() + _plain_drop(s["x"].float(), s["kw"])
    y = h * (h.square().mean(-1, keepdim=True) + s["kw"]["eps"]).rsqrt() * s["weight"]
    h = h.to(s["x"].dtype)
    if not s["case"]["bits"]:
        return y.to(s["x"].dtype), h
    top = y.abs().amax(1, keepdim=True)
    codes = (y * torch.where(top > 0, FLOAT8_MAX / top, 0.0)).clamp(-FLOAT8_MAX, FLOAT8_MAX).to(torch.float8_e4m3fn)
    return codes, top[:, 0] / FLOAT8_MAX, h


def _plain_norm_bwd(s):
    h, w = s["h"].float(), s["weight"]
    rstd = (h.square().mean(-1, keepdim=True) + s["kw"]["eps"]).rsqrt()
    unit = h * rstd
    g = s["grad_y"].float()
    grad_w = (g * unit).sum(0, dtype=torch.float64).float()
    g = g * w
    grad = s["grad_h"].float() + rstd * (g - unit * (g * unit).mean(-1, keepdim=True))
    return _plain_drop(grad, s["kw"]).to(s["h"].dtype), grad.to(s["h"].dtype), grad_w


def run(s):
    op = s["case"]["op"]
    if not own:
        if op == "attention_fwd":
            return _plain_attention_fwd(s)
        if op == "attention_bwd":
            return _plain_attention_bwd(s)
        if op == "dropout_fwd":
            return _plain_dropout_fwd(s)
        if op == "dropout_bwd":
            return _plain_drop(s["x"].float(), s["kw"]).to(s["x"].dtype)
        return _plain_norm_fwd(s) if op == "norm_fwd" else _plain_norm_bwd(s)

    import paper_2202_00441_b200 as fb

    case, kw = s["case"], s["kw"]
    if op.startswith("attention"):
        if "table" in s:
            bias = fb.fewbit_relative_bias_fwd(s["table"], case["max_distance"], bidirectional=case["both"])
            kw = {**kw, "distance_bias": bias}
        if op == "attention_fwd":
            return fb.fewbit_attention_fwd(s["q"], s["k"], s["v"], **kw)
        grads = fb.fewbit_attention_bwd(s["grad_out"], s["q"], s["k"], s["v"], s["out"], s["lse"], **kw)
        if "table" in s:
            return (*grads[:3], fb.fewbit_relative_bias_bwd(grads[3], s["table"], bidirectional=case["both"]))
        return grads
    if op == "dropout_fwd":
        return fb.fewbit_dropout_fwd(s["x"], residual=s["residual"], **kw)
    if op == "dropout_bwd":
        return fb.fewbit_dropout_bwd(s["x"], **kw)
    if op == "norm_fwd":
        return fb.fewbit_add_rms_norm_fwd(s["x"], s["residual"], s["weight"], bits=case["bits"] or None, **kw)
    grad_x, grad_residual, grad_weight = fb.fewbit_add_rms_norm_bwd(s["grad_y"], s["grad_h"], s["h"], s["weight"], **kw)
    return grad_x, grad_residual, grad_weight


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without, and its outputs in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def _seen_keys(i, keys, first_key, case, shift, prefix):
    """How many of `keys` keys from first_key on row i sees by order."""
    if not case["causal"]:
        return keys
    return max(0, min(keys, max(i + 1 + shift, prefix) - first_key))


def _seen_pairs(case):
    """(row, key) pairs that the masks leave, over the batch."""
    shift, total = case["k_len"] - case["q_len"], 0
    prefixes = _prefixes(case) if case["prefix"] else [0] * case["batch"]
    for b in range(case["batch"]):
        spans = [(0, case["q_len"], 0, case["k_len"])]
        if case["docs"]:
            q, k = _cuts(case, b), _key_cuts(case, b)
            spans = list(zip(q, q[1:], k, k[1:]))
        for q0, q1, k0, k1 in spans:
            if case["causal"]:
                total += sum(_seen_keys(i, k1 - k0, k0, case, shift, prefixes[b]) for i in range(q0, q1))
            else:
                total += (q1 - q0) * (k1 - k0)
    return total


def work(case):
    op, e = case["op"], BYTES[case["dtype"]]
    if op.startswith("attention"):
        q = case["batch"] * case["q_len"] * case["heads"] * case["head_dim"] * e
        k = case["batch"] * case["k_len"] * case["kv_heads"] * case["head_dim"] * e
        rows = case["batch"] * case["q_len"] * case["heads"] * 4
        ids = 4 * case["batch"] * (case["q_len"] + case["k_len"]) if case["docs"] else 0
        table = case["buckets"] * case["heads"] * BYTES[case["table"]]
        pair = 2 * _seen_pairs(case) * case["heads"] * case["head_dim"]
        if op == "attention_fwd":                                # q, k, v in; out and lse out; two products
            return {"bytes": 2 * q + 2 * k + rows + ids + table, "flops": 2 * pair}
        return {"bytes": 4 * q + 4 * k + rows + ids + 2 * table, "flops": 5 * pair}   # five products; the scores are recomputed
    n = case["rows"] * case["width"]
    if op.startswith("dropout"):
        return {"bytes": n * e * (3 if case["residual"] else 2), "flops": 2 * n}
    if op == "norm_fwd":                                         # branch and residual in; stream and result out
        out = n + 4 * case["rows"] if case["bits"] else n * e
        return {"bytes": 3 * n * e + out + 4 * case["width"], "flops": 6 * n}
    # both gradients and the stream in; the branch's and the residual's gradients out (one and the same without dropout)
    return {"bytes": n * e * (5 if case["p"] else 4) + 8 * case["width"], "flops": 12 * n}


def _exact_bucket(d, buckets, most, both):
    """One distance's bucket, in whole numbers: the logarithm's borders are compared as powers."""
    n = buckets // 2 if both else buckets
    far = abs(d) if both else max(-d, 0)
    half = n // 2
    if far < half:
        found = far
    else:
        step = 0                                                 # (far / half) ** (n - half) >= (most / half) ** (step + 1)
        while step < n - half - 1 and far ** (n - half) * half ** (step + 1) >= most ** (step + 1) * half ** (n - half):
            step += 1
        found = half + step
    return found + n if both and d > 0 else found


def _exact_attention(s, case):
    dev, kw = s["q"].device, s["kw"]
    backward = case["op"] == "attention_bwd"
    h, hk, d, lq, lk = (case[x] for x in ("heads", "kv_heads", "head_dim", "q_len", "k_len"))
    group, most = h // hk, case["max_distance"]
    away = torch.arange(lk, device=dev).view(1, -1) - torch.arange(lq, device=dev).view(-1, 1) - (lk - lq)
    bucket = None
    if case["buckets"]:
        of = torch.tensor([_exact_bucket(x, case["buckets"], most, case["both"]) for x in range(-most, most + 1)], device=dev)
        bucket = of[away.clamp(-most, most) + most]
    if backward:
        out = [torch.zeros(s[n].shape, dtype=torch.float64, device=dev) for n in ("q", "k", "v")]
        if case["buckets"]:
            out.append(torch.zeros(case["buckets"], h, dtype=torch.float64, device=dev))
    else:
        out = [torch.zeros(s["q"].shape, dtype=torch.float64, device=dev), torch.zeros(case["batch"], h, lq, dtype=torch.float64, device=dev)]
    for b in range(case["batch"]):
        hidden = torch.zeros(lq, lk, dtype=torch.bool, device=dev)
        if case["causal"]:
            hidden |= away > 0
            if case["prefix"]:
                hidden[:, :int(kw["prefix_lens"][b])] = False
        if case["docs"]:
            hidden |= kw["q_documents"][b].view(-1, 1) != kw["k_documents"][b].view(1, -1)
        for i in range(h):
            q, k, v = s["q"][b, :, i].double(), s["k"][b, :, i // group].double(), s["v"][b, :, i // group].double()
            z = q @ k.T / math.sqrt(d)
            slope = None
            if case["cap"]:
                z.div_(case["cap"]).tanh_()
                slope = 1 - z * z if backward else None
                z.mul_(case["cap"])
            if case["slopes"]:
                z.sub_(kw["slopes"][i].double() * away.abs())
            if bucket is not None:
                z.add_(s["table"][:, i].double()[bucket])
            z.masked_fill_(hidden, -math.inf)
            lse = torch.logsumexp(z, 1)
            p = z.sub_(lse[:, None]).exp_().nan_to_num_(nan=0.0)
            if not backward:
                out[0][b, :, i] = p @ v
                out[1][b, i] = lse
                continue
            g = s["grad_out"][b, :, i].double()
            out[2][b, :, i // group] += p.T @ g
            dz = g @ v.T
            dz.sub_((p * dz).sum(1, keepdim=True)).mul_(p)
            if bucket is not None:
                for x in range(case["buckets"]):
                    out[3][x, i] += dz[bucket == x].sum()
            if slope is not None:
                dz.mul_(slope)
            dz.div_(math.sqrt(d))
            out[0][b, :, i] = dz @ k
            out[1][b, :, i // group] += dz.T @ q
    return tuple(out)


def _exact_kept(n, case, kw, dev):
    """Which of n elements dropout keeps; the generator's words as pairs of 16-bit halves."""
    e = torch.arange(-(-n // 4), device=dev)
    c0, c1, c2, c3 = e % 2 ** 32, e // 2 ** 32, torch.full_like(e, kw["place"]), torch.zeros_like(e)
    k0, k1 = kw["seed"] % 2 ** 32, kw["seed"] // 2 ** 32

    def times(x, m):
        parts = [(x // 2 ** 16) * (m // 2 ** 16), (x // 2 ** 16) * (m % 2 ** 16), (x % 2 ** 16) * (m // 2 ** 16), (x % 2 ** 16) * (m % 2 ** 16)]
        middle = parts[1] % 2 ** 16 + parts[2] % 2 ** 16 + parts[3] // 2 ** 16
        return parts[0] + parts[1] // 2 ** 16 + parts[2] // 2 ** 16 + middle // 2 ** 16, (middle % 2 ** 16) * 2 ** 16 + parts[3] % 2 ** 16

    for i in range(10):
        a, b = times(c0, PHILOX_MULTIPLIERS[0]), times(c2, PHILOX_MULTIPLIERS[1])
        r0, r1 = (k0 + i * PHILOX_KEYS[0]) % 2 ** 32, (k1 + i * PHILOX_KEYS[1]) % 2 ** 32
        c0, c1, c2, c3 = b[0] ^ c1 ^ r0, b[1], a[0] ^ c3 ^ r1, a[1]
    words = torch.empty(len(e), 4, dtype=torch.int64, device=dev)
    words[:, 0], words[:, 1], words[:, 2], words[:, 3] = c0, c1, c2, c3
    return words.view(-1)[:n] >= int(math.floor(kw["p"] * 2 ** 32 + 0.5))


def _exact_drop(x, case, kw):
    if case["p"] == 0:
        return x
    return x * _exact_kept(x.numel(), case, kw, x.device).view_as(x) / (1 - case["p"])


def _exact_rows(s, case):
    kw = s["kw"]
    if case["op"].startswith("dropout"):
        y = _exact_drop(s["x"].double(), case, kw)
        return y if s["residual"] is None else y + s["residual"].double()
    w = s["weight"].double()
    if case["op"] == "norm_fwd":
        h = s["residual"].double() + _exact_drop(s["x"].double(), case, kw)
        y = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + kw["eps"]) * w
        if case["bits"]:
            top = y.abs().max(1).values
            return y * (448 / top).view(-1, 1), top / 448, h     # what the codes stand for, before they are rounded
        return y, h
    h, g = s["h"].double(), s["grad_y"].double()
    norm = torch.sqrt(h.pow(2).mean(1, keepdim=True) + kw["eps"])
    grad_w = (g * h / norm).sum(0)
    g = g * w
    grad = s["grad_h"].double() + g / norm - h * (g * h).mean(1, keepdim=True) / norm ** 3
    return _exact_drop(grad, case, kw), grad, grad_w


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("attention"):
        products = 10 * case["batch"] * case["q_len"] * case["k_len"] * case["heads"] * case["head_dim"]
        if products > 1e14:
            return None
        return _exact_attention(s, case)
    return _exact_rows(s, case)
