"""Workloads for timing the training and answering operators of a decoder block with an encoder:
LayerNorm over rows (forward, backward), the global gradient norm with clipping, and cross
attention to states of another length (forward, single tokens, backward).

``own`` False computes a case from elementary torch operations in 32 bits; ``own`` True calls the
library's entry points.  Both take what ``prepare`` returns.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_CODES = {"fp32": 0, "bf16": 1, "fp16": 2}
_EPS = 1e-5
_CLIP_EPS = 1e-6


# ------------------------------------------------------------------ cases --
def listed():
    return [
        # the normalisation before a block while eight sequences each produce a token
        dict(name="ln_fwd_tokens", op="ln_fwd", rows=8, n=1024, dtype="bf16", params="bf16"),
        # the same layer over a training batch: 8 sequences of 2048 tokens
        dict(name="ln_fwd_batch", op="ln_fwd", rows=16384, n=4096, dtype="bf16", params="fp32"),
        # odd width in full precision, as in a small model's fine-tuning run
        dict(name="ln_bwd_odd", op="ln_bwd", rows=2999, n=1537, dtype="fp32", params="fp32"),
        # gradient of the normalisation over a training batch
        dict(name="ln_bwd_batch", op="ln_bwd", rows=16384, n=4096, dtype="bf16", params="fp32"),
        # clipping the gradients of a two-layer model of width 512: launch latency counts
        dict(name="clip_small", op="clip", layers=2, width=512, vocab=1000, dtype="mixed"),
        # clipping a model of 24 layers, some 400 million gradients in 16 bits
        dict(name="clip_large", op="clip", layers=24, width=1152, vocab=20011, dtype="bf16"),
        # the paper's attention task (512 queries, 16 heads of 32) read across to 1000 states
        dict(name="xattn_fwd_small", op="xattn_fwd", batch=1, q_rows=512, kv_rows=1000, heads=16, kv_heads=16,
             dim=32, dtype="bf16", ragged=False, fused_kv=False),
        # a training batch: four targets of 2048 tokens against padded sources of up to 4096
        dict(name="xattn_fwd_batch", op="xattn_fwd", batch=4, q_rows=2048, kv_rows=4096, heads=16, kv_heads=16,
             dim=128, dtype="bf16", ragged=True, fused_kv=False),
        # one token for each of sixteen sequences against 1500 states
        dict(name="xattn_token", op="xattn_token", batch=16, q_rows=1, kv_rows=1500, heads=16, kv_heads=16,
             dim=64, dtype="fp16", ragged=True, fused_kv=True),
        # one token each against long sources, four query heads to a key head
        dict(name="xattn_token_long", op="xattn_token", batch=8, q_rows=1, kv_rows=16384, heads=32, kv_heads=8,
             dim=128, dtype="bf16", ragged=False, fused_kv=False),
        # gradient of a short ragged batch with shared key heads
        dict(name="xattn_bwd_small", op="xattn_bwd", batch=2, q_rows=100, kv_rows=333, heads=8, kv_heads=4,
             dim=64, dtype="fp16", ragged=True, fused_kv=True),
        # gradient of the training batch
        dict(name="xattn_bwd_batch", op="xattn_bwd", batch=4, q_rows=2048, kv_rows=4096, heads=16, kv_heads=16,
             dim=128, dtype="bf16", ragged=True, fused_kv=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "clip", "xattn_fwd", "xattn_token", "xattn_bwd"])
    if op in ("ln_fwd", "ln_bwd"):
        n = _log_int(rng, 32, 12000)
        rows = _log_int(rng, 1, max(2, min(20000, (1 << 26) // n)))
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        params = rng.choice([dtype, "fp32"])
        if dtype == "fp32":
            rows = max(1, rows // 2)
        return dict(op=op, rows=rows, n=n, dtype=dtype, params=params)
    if op == "clip":
        return dict(op=op, layers=rng.randint(1, 20), width=_log_int(rng, 30, 1000), vocab=_log_int(rng, 100, 20000),
                    dtype=rng.choice(["bf16", "fp16", "fp32", "mixed"]))
    dtype = rng.choice(["bf16", "fp16"])
    dim = rng.choice([32, 64, 64, 80, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 16])
    group = rng.choice([1, 1, 2, 4]) if kv_heads <= 8 else 1
    batch = _log_int(rng, 1, 16)
    if op == "xattn_token":
        rows = rng.choice([1, 1, 1, 2, 4])
        kv_rows = _log_int(rng, 16, 20000)
        while batch * kv_heads * kv_rows * dim > (1 << 27):
            kv_rows //= 2
    else:
        rows = _log_int(rng, 1, 3000)
        kv_rows = _log_int(rng, 1, 5000)
        while batch * kv_heads * group * rows * kv_rows * dim > (1 << 36):
            batch, rows = max(1, batch // 2), max(1, rows - rows // 4)
    return dict(op=op, batch=batch, q_rows=rows, kv_rows=kv_rows, heads=kv_heads * group, kv_heads=kv_heads, dim=dim,
                dtype=dtype, ragged=rng.random() < 0.5, fused_kv=rng.random() < 0.5)


def _clip_shapes(case):
    """(elements, type) of every gradient: a layer's matrices, biases and norms, then the embedding."""
    w, t = case["width"], case["dtype"]
    mat, vec = ("bf16", "fp32") if t == "mixed" else (t, t)
    out = []
    for _ in range(case["layers"]):
        out += [(w, vec), (w, vec), (3 * w * w, mat), (3 * w, vec), (w * w, mat), (w, vec),
                (w, vec), (w, vec), (4 * w * w, mat), (4 * w, vec), (4 * w * w, mat), (w, vec)]
    return out + [(case["vocab"] * w, mat), (w, vec), (w, vec)]


def _lens(case):
    """Valid states of each batch item: all of them, or between three eighths and all."""
    b, n = case["batch"], case["kv_rows"]
    return [max(1, n - (i * n * 5) // (8 * b)) if case["ragged"] else n for i in range(b)]


def work(case):
    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        rows, n, es, ps = case["rows"], case["n"], _BYTES[case["dtype"]], _BYTES[case["params"]]
        if op == "ln_fwd":
            return {"bytes": 2 * rows * n * es + 2 * n * ps + 8 * rows, "flops": 8 * rows * n}
        return {"bytes": 3 * rows * n * es + 3 * n * ps + 8 * rows, "flops": 14 * rows * n}
    if op == "clip":
        shapes = _clip_shapes(case)
        return {"bytes": sum(2 * n * _BYTES[t] for n, t in shapes) + 4, "flops": 3 * sum(n for n, _ in shapes)}
    b, lq, hq, hk, d = (case[k] for k in ("batch", "q_rows", "heads", "kv_heads", "dim"))
    keys, es = sum(_lens(case)), _BYTES[case["dtype"]]
    q_bytes, kv_bytes, lse = b * lq * hq * d * es, keys * hk * d * es, 4 * b * lq * hq
    pairs = lq * keys * hq * d
    if op == "xattn_token":
        return {"bytes": 2 * q_bytes + 2 * kv_bytes, "flops": 4 * pairs}
    if op == "xattn_fwd":
        return {"bytes": 2 * q_bytes + 2 * kv_bytes + lse, "flops": 4 * pairs}
    full = b * case["kv_rows"] * hk * d * es
    return {"bytes": 4 * q_bytes + 2 * kv_bytes + 2 * full + lse, "flops": 10 * pairs}


# ----------------------------------------------------------------- inputs --
def _buckets(case):
    """One flat buffer per type, and every gradient of the case as a part of it."""
    shapes = _clip_shapes(case)
    total = {}
    for n, t in shapes:
        total[t] = total.get(t, 0) + n
    buckets = {t: torch.empty(n, dtype=_TYPES[t], device="cuda") for t, n in total.items()}
    used, parts = dict.fromkeys(total, 0), []
    for n, t in shapes:
        parts.append(buckets[t][used[t]:used[t] + n])
        used[t] += n
    return list(buckets.values()), parts


def _inputs(case, seed):
    """The tensors of a case from the seed alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)

    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        rows, n, t, p = case["rows"], case["n"], _TYPES[case["dtype"]], _TYPES[case["params"]]
        # activations: rows of different mean and spread
        x = (normal(rows, n) * (0.5 + 2 * torch.rand(rows, 1, generator=gen, device="cuda")) + normal(rows, 1)).to(t)
        s = dict(x=x, gamma=(1 + 0.1 * normal(n)).to(p), beta=(0.1 * normal(n)).to(p))
        if op == "ln_bwd":
            xf = x.float()
            mean = xf.mean(1)
            s["mean"] = mean
            s["rstd"] = torch.rsqrt((xf - mean[:, None]).square().mean(1) + _EPS)
            s["dy"] = normal(rows, n).mul_(0.1).to(t)
        return s
    if op == "clip":
        # gradients whose size differs from tensor to tensor, lying one behind the other in a bucket per type;
        # the norm is well above the limit
        buckets, grads = _buckets(case)
        for i, g in enumerate(grads):
            g.copy_(normal(g.numel()).mul_(10.0 ** (-2 - 2 * (i % 7) / 6)))
        return dict(buckets=buckets, grads=grads)
    b, lq, lk, hq, hk, d = (case[k] for k in ("batch", "q_rows", "kv_rows", "heads", "kv_heads", "dim"))
    t = _TYPES[case["dtype"]]
    s = dict(q=normal(b, lq, hq, d).mul_(1.5).to(t))
    if case["fused_kv"]:                       # one projection wrote keys and values side by side
        kv = normal(b, lk, 2, hk, d).to(t)
        s["kv"], s["k"], s["v"] = kv, kv[:, :, 0], kv[:, :, 1]
    else:
        s["k"], s["v"] = normal(b, lk, hk, d).to(t), normal(b, lk, hk, d).to(t)
    s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")
    if op == "xattn_bwd":
        o, lse = _xattn_forward(case, s)
        s["o"], s["lse"], s["do"] = o, lse, normal(b, lq, hq, d).mul_(0.1).to(t)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    op = case["op"]
    # the buffers that the results go to
    if op == "ln_fwd":
        s["y"] = torch.empty_like(s["x"])
        s["mean"] = torch.empty(case["rows"], device="cuda")
        s["rstd"] = torch.empty(case["rows"], device="cuda")
    elif op == "ln_bwd":
        s["dx"] = torch.empty_like(s["x"])
        s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
    elif op == "clip":
        s["out_buckets"], s["out"] = _buckets(case)
        s["norm"] = torch.empty(1, device="cuda")
    else:
        s["out"] = torch.empty_like(s["q"])
        if op == "xattn_fwd":
            s["out_lse"] = torch.empty(case["batch"], case["heads"], case["q_rows"], device="cuda")
        elif op == "xattn_bwd":
            if case["fused_kv"]:
                dkv = torch.empty_like(s["kv"])
                s["dk"], s["dv"] = dkv[:, :, 0], dkv[:, :, 1]
            else:
                s["dk"], s["dv"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a user's program sets up once: sizes, strides, tables of tensors, scratch."""
    from paper_2506_09092_b200 import binding as lib
    case = s["case"]
    op = case["op"]
    s["lib"] = lib
    nbytes = 0
    if op == "ln_bwd":
        nbytes = lib.layernorm_rows_bwd_scratch_bytes(case["rows"], case["n"])
    elif op == "clip":
        s["table"] = lib.tensor_table(s["grads"], s["out"])
        nbytes = lib.grad_norm_scratch_bytes(s["table"])
    elif op.startswith("xattn"):
        s["shape"] = lib.XattnShape.of(s["q"], s["k"], s["v"], s["out"])
        nbytes = (lib.xattn_bwd_scratch_bytes if op == "xattn_bwd" else lib.xattn_fwd_scratch_bytes)(s["shape"])
    s["scratch"] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    s["scratch_bytes"] = nbytes


# ------------------------------------------------------------------- runs --
def run(s):
    if own:
        return _run_own(s)
    return _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    if "lib" not in s:
        _plan(s)
    lib, case = s["lib"], s["case"]
    op, stream = case["op"], torch.cuda.current_stream()
    if op == "ln_fwd":
        n = case["n"]
        lib.layernorm_rows(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], case["rows"], n, n, n,
                           _CODES[case["dtype"]], _CODES[case["params"]], _EPS, stream)
        return s["y"], s["mean"], s["rstd"]
    if op == "ln_bwd":
        n = case["n"]
        lib.layernorm_rows_bwd(s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"],
                               case["rows"], n, n, n, n, _CODES[case["dtype"]], _CODES[case["params"]],
                               s["scratch"], s["scratch_bytes"], stream)
        return s["dx"], s["dgamma"], s["dbeta"]
    if op == "clip":
        lib.grad_clip_norm(s["table"], 1.0, _CLIP_EPS, s["norm"], s["scratch"], s["scratch_bytes"], stream)
        return [s["norm"]] + s["out_buckets"]
    if op == "xattn_bwd":
        lib.xattn_bwd(s["shape"], s["q"], s["k"], s["v"], s["lens"], s["o"], s["lse"], s["do"],
                      s["out"], s["dk"], s["dv"], s["scratch"], s["scratch_bytes"], stream)
        return s["out"], s["dk"], s["dv"]
    lse = s.get("out_lse")
    lib.xattn_fwd(s["shape"], s["q"], s["k"], s["v"], s["lens"], s["out"], lse,
                  s["scratch"], s["scratch_bytes"], stream)
    return s["out"] if lse is None else (s["out"], lse)


def _ln_fwd(s):
    x = s["x"].float()
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = torch.rsqrt(xc.square().mean(1) + _EPS)
    y = xc * rstd[:, None] * s["gamma"].float() + s["beta"].float()
    return y.to(s["x"].dtype), mean, rstd


def _ln_bwd(s):
    x, dy = s["x"].float(), s["dy"].float()
    xhat = (x - s["mean"][:, None]) * s["rstd"][:, None]
    dgamma, dbeta = (dy * xhat).sum(0), dy.sum(0)
    g = dy * s["gamma"].float()
    dx = (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True)) * s["rstd"][:, None]
    p = s["gamma"].dtype
    return dx.to(s["x"].dtype), dgamma.to(p), dbeta.to(p)


def _clip(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        total += g.float().square().sum(dtype=torch.float64)
    norm = total.sqrt()
    coef = (1.0 / (norm + _CLIP_EPS)).clamp(max=1.0).float()
    return [norm.float().reshape(1)] + [(g.float() * coef).to(g.dtype) for g in s["buckets"]]


def _heads_first(case, s):
    """q, k, v as (batch, heads, rows, dim) in 32 bits, key heads repeated, and the mask of padded states."""
    rep = case["heads"] // case["kv_heads"]
    q = s["q"].float().transpose(1, 2)
    k = s["k"].float().transpose(1, 2).repeat_interleave(rep, 1)
    v = s["v"].float().transpose(1, 2).repeat_interleave(rep, 1)
    pad = torch.arange(case["kv_rows"], device="cuda")[None, :] >= s["lens"][:, None]
    return q, k, v, pad[:, None, None, :]


def _xattn_forward(case, s):
    q, k, v, pad = _heads_first(case, s)
    scores = torch.matmul(q, k.transpose(2, 3)) * (case["dim"] ** -0.5)
    scores = scores.masked_fill_(pad, float("-inf"))
    top = scores.amax(3, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / total
    return o.transpose(1, 2).contiguous().to(s["q"].dtype), (top + total.log()).squeeze(3)


def _xattn_fwd(s):
    return _xattn_forward(s["case"], s)


def _xattn_token(s):
    return _xattn_forward(s["case"], s)[0]


def _xattn_bwd(s):
    case = s["case"]
    b, lk, hk, d = case["batch"], case["kv_rows"], case["kv_heads"], case["dim"]
    q, k, v, pad = _heads_first(case, s)
    scale = d ** -0.5
    do, o = s["do"].float().transpose(1, 2), s["o"].float().transpose(1, 2)
    delta = (do * o).sum(3, keepdim=True)
    p = (torch.matmul(q, k.transpose(2, 3)) * scale - s["lse"][..., None]).exp_().masked_fill_(pad, 0.0)
    dv = torch.matmul(p.transpose(2, 3), do)
    ds = torch.matmul(do, v.transpose(2, 3)).sub_(delta).mul_(p).mul_(scale)
    del p
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), q)
    dk, dv = (g.reshape(b, hk, -1, lk, d).sum(2).transpose(1, 2).to(s["q"].dtype) for g in (dk, dv))
    return dq.transpose(1, 2).to(s["q"].dtype), dk, dv


_PLAIN = dict(ln_fwd=_ln_fwd, ln_bwd=_ln_bwd, clip=_clip, xattn_fwd=_xattn_fwd, xattn_token=_xattn_token,
              xattn_bwd=_xattn_bwd)


# ------------------------------------------------------------------ exact --
def exact(case, seed):
    """The operators' definitions in 64 bits, one row block, tensor or head at a time."""
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("ln_fwd", "ln_bwd"):
        n = case["n"]
        gamma, beta = s["gamma"].double(), s["beta"].double()
        first, dgamma, dbeta, means, rstds = [], torch.zeros_like(gamma), torch.zeros_like(gamma), [], []
        step = max(1, (1 << 25) // n)
        for r in range(0, case["rows"], step):
            x = s["x"][r:r + step].double()
            if op == "ln_fwd":
                mean = x.sum(1, keepdim=True) / n
                rstd = 1.0 / (((x - mean) ** 2).sum(1, keepdim=True) / n + _EPS).sqrt()
                first.append((x - mean) * rstd * gamma + beta)
                means.append(mean[:, 0])
                rstds.append(rstd[:, 0])
            else:
                rstd = s["rstd"][r:r + step].double()[:, None]
                z = (x - s["mean"][r:r + step].double()[:, None]) * rstd
                dy = s["dy"][r:r + step].double()
                g = dy * gamma
                first.append(rstd * (g - g.sum(1, keepdim=True) / n - z * ((g * z).sum(1, keepdim=True) / n)))
                dgamma += (dy * z).sum(0)
                dbeta += dy.sum(0)
        if op == "ln_fwd":
            return torch.cat(first), torch.cat(means), torch.cat(rstds)
        return torch.cat(first), dgamma, dbeta
    if op == "clip":
        norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["grads"]))
        coef = min(1.0, 1.0 / (norm + _CLIP_EPS))
        return [torch.tensor([norm], dtype=torch.float64, device="cuda")] + [g.double() * coef for g in s["buckets"]]
    b, lq, hq, hk, d = (case[k] for k in ("batch", "q_rows", "heads", "kv_heads", "dim"))
    scale = 1.0 / math.sqrt(d)
    out = torch.zeros(b, lq, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(b, hq, lq, dtype=torch.float64, device="cuda")
    dk = torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") if op == "xattn_bwd" else None
    dv = torch.zeros_like(dk) if op == "xattn_bwd" else None
    for i, keys in enumerate(_lens(case)):
        for h in range(hq):
            kh = h * hk // hq
            k, v, q = s["k"][i, :keys, kh].double(), s["v"][i, :keys, kh].double(), s["q"][i, :, h].double()
            z = scale * (q @ k.T)
            if op != "xattn_bwd":
                lse[i, h] = torch.logsumexp(z, 1)
                out[i, :, h] = torch.exp(z - lse[i, h][:, None]) @ v
                continue
            p = torch.exp(z - s["lse"][i, h].double()[:, None])
            do = s["do"][i, :, h].double()
            delta = (do * s["o"][i, :, h].double()).sum(1, keepdim=True)
            ds = p * (do @ v.T - delta)
            out[i, :, h] = scale * (ds @ k)
            dk[i, :keys, kh] += scale * (ds.T @ q)
            dv[i, :keys, kh] += p.T @ do
    if op == "xattn_bwd":
        return out, dk, dv
    return out if op == "xattn_token" else (out, lse)
