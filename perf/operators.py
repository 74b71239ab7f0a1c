"""Attention over token sequences and rotary positions: the cases, their plain forms and the library's calls.

The sequences ("documents") of a batch are packed one behind the other, as the graphs of a batch are: rows [T, heads, d],
document g owns rows cu_seqlens[g] .. cu_seqlens[g + 1] - 1, and a token's position is its index within its document.

  fwd      gt_position_attn_fwd: out = softmax(S) v and the rows' log-sum-exp, with
           S_ij = cap tanh(x_ij / cap) - slopes[h] |i - j|,  x_ij = q_i . k_j / sqrt(d)   (cap 0: x_ij itself; no slopes: no term)
           over the keys j of query i's document, those after i only where they belong to the document's prefix (causal)
  train    the forward and gt_position_attn_bwd: one training step of the layer
  rotary   gt_rotary: rotation of pairs of channels of q and k by position x frequency
  inverse  gt_rotary the other way: the gradient of the rotation

Fields: `documents` documents of `n_min` to `n_max` tokens, whose lengths follow from `lengths`; `heads` query heads that share
`kv_heads` key heads of `head_dim` channels; `fused`: q, k and v are parts of the rows of one projection; `spread`: standard
deviation of the scores x.  fwd, train: `causal`, `prefix` (share of a document, at most, that all its tokens see), `slopes`, `cap`.
rotary, inverse: `rot_dim` channels of a head are rotated, `interleaved` pairs or halves, `positions` (0: a token's own, else
random ones up to it), `scale`, `dtype`.
"""
import math
import random

import torch

own = False
ROWS_AT_A_TIME = 1 << 27          # scores of a step of the plain forms
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _attn(what, documents, n_min, n_max, heads, kv_heads, head_dim, causal=True, prefix=0.0, slopes=False, cap=0.0, spread=1.0,
          fused=False, lengths=0):
    return {"what": what, "documents": documents, "n_min": n_min, "n_max": n_max, "lengths": lengths, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "prefix": prefix, "slopes": slopes, "cap": cap,
            "spread": spread, "fused": fused}


def _rotary(what, documents, n_min, n_max, heads, kv_heads, head_dim, rot_dim, interleaved, dtype, positions=0, scale=1.0,
            fused=False, lengths=0):
    return {"what": what, "documents": documents, "n_min": n_min, "n_max": n_max, "lengths": lengths, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "rot_dim": rot_dim, "interleaved": interleaved, "dtype": dtype,
            "positions": positions, "scale": scale, "fused": fused}


def listed():
    cases = {
        # The smallest calls: one short sequence with few, narrow heads.  Launches and host work count here.
        "fwd_256": _attn("fwd", 1, 256, 256, 4, 4, 32),
        "train_256": _attn("train", 1, 256, 256, 4, 4, 32),
        # Inference on a packed batch of ragged documents, with the linear penalty on distance.
        "fwd_docs64": _attn("fwd", 64, 512, 2048, 16, 16, 64, slopes=True),
        # A prefix model with capped scores and shared key heads, reading its fused projection.
        "fwd_prefix_4096": _attn("fwd", 4, 4096, 4096, 8, 2, 64, prefix=0.5, cap=30.0, spread=4.0, fused=True),
        # An encoder: every token sees the whole long sequence.
        "fwd_full_16384": _attn("fwd", 1, 16384, 16384, 8, 8, 64, causal=False),
        # One training step of an ordinary sequence.
        "train_4096": _attn("train", 1, 4096, 4096, 8, 8, 64),
        # One training step of a packed batch of ragged documents with all that the operator offers.
        "train_docs64": _attn("train", 64, 512, 2048, 16, 4, 64, prefix=0.3, slopes=True, cap=50.0, spread=3.0, fused=True),
        # One training step of one long document.
        "train_32768": _attn("train", 1, 32768, 32768, 8, 8, 64, slopes=True),
        # Positions of one new token of each of a few sequences, far into them: latency.
        "rotary_tokens": _rotary("rotary", 8, 1, 1, 8, 2, 64, 64, False, "bf16", positions=1 << 20),
        # The packed batch of ragged documents, in the rows of the fused projection, half of each head.
        "rotary_docs64": _rotary("rotary", 64, 512, 2048, 16, 4, 64, 32, False, "bf16", fused=True),
        # Rows of many long sequences in pairs of neighbours, with the factor of a scaled context.
        "rotary_long": _rotary("rotary", 4, 65536, 65536, 8, 8, 64, 64, True, "fp16", positions=1 << 24, scale=1.1),
        # The gradient's way back, in fp32.
        "inverse_32768": _rotary("inverse", 3, 10000, 32768, 8, 8, 32, 32, False, "fp32"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _between(rng, low, high):
    """A whole number whose logarithm is spread evenly."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    what = rng.choice(("fwd", "train", "fwd", "train", "rotary", "inverse"))
    documents = rng.choice((1, 1, _between(rng, 2, 200)))
    head_dim = rng.choice((32, 64, 64))
    kv_heads = rng.choice((1, 2, 4, 8))
    heads = kv_heads * rng.choice((1, 1, 2, 3, 4) if kv_heads < 8 else (1, 2))
    fused = rng.random() < 0.3
    lengths = rng.randint(1, 1 << 30)
    if what in ("rotary", "inverse"):
        top = max(2, min(65536, (1 << 18) // documents * 8 // (heads + kv_heads)))
        n_max = _between(rng, 2, top)
        return _rotary(what, documents, max(1, n_max // rng.randint(1, 8)), n_max, heads, kv_heads, head_dim,
                       rng.choice((head_dim, head_dim // 2, 16)), rng.random() < 0.5, rng.choice(("bf16", "bf16", "fp16", "fp32")),
                       rng.choice((0, 0, 1 << rng.randint(10, 26))), rng.choice((1.0, 1.0, 1.25)), fused, lengths)
    n_max = _between(rng, 16, min(16384, 100000 // documents))
    causal = rng.random() < 0.75
    cap = rng.choice((0.0, 0.0, 30.0, 50.0))
    return _attn(what, documents, max(1, n_max // rng.randint(1, 8)), n_max, heads, kv_heads, head_dim, causal,
                 rng.choice((0.0, 0.0, 0.4, 1.0)) if causal else 0.0, rng.random() < 0.4, cap, rng.choice((1.0, 2.0, 4.0)), fused, lengths)


def _lengths(case):
    r = random.Random(case["lengths"])
    return [r.randint(case["n_min"], case["n_max"]) for _ in range(case["documents"])]


def _prefixes(case):
    r = random.Random(case["lengths"] + 1)
    return [int(n * case["prefix"] * r.random()) for n in _lengths(case)]


def _inputs(case, seed):
    """The same for everybody: what a layer has in hand before the call."""
    dev = torch.device("cuda", torch.cuda.current_device())
    rng = torch.Generator(device=dev).manual_seed(seed)
    sizes, H, G, d = _lengths(case), case["heads"], case["kv_heads"], case["head_dim"]
    T = sum(sizes)
    ends = torch.tensor([0] + sizes).cumsum(0)
    rotary = case["what"] in ("rotary", "inverse")
    dtype = DTYPES[case["dtype"]] if rotary else torch.bfloat16
    rows = torch.empty(T, H + 2 * G, d, dtype=dtype, device=dev) if case["fused"] else None

    def normal(at, heads, std=1.0):
        x = (torch.randn(T, heads, d, device=dev, generator=rng) * std).to(dtype)
        if rows is None or at < 0:
            return x
        rows[:, at:at + heads] = x
        return rows[:, at:at + heads]

    s = {"case": case, "sizes": sizes, "ends": ends.tolist(), "cu_seqlens": ends.to(device=dev, dtype=torch.int32)}
    s["q"], s["k"] = normal(0, H, case.get("spread", 1.0)), normal(H, G)
    if rotary:
        s["frequencies"] = torch.tensor([10000.0 ** (-2.0 * i / case["rot_dim"]) for i in range(case["rot_dim"] // 2)],
                                        dtype=torch.float64, device=dev)
        s["positions"] = torch.randint(0, case["positions"], (T,), device=dev, generator=rng, dtype=torch.int32) if case["positions"] else None
        return s
    s["v"], s["dout"] = normal(H + G, G), normal(-1, H)
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device=dev) if case["slopes"] else None
    s["prefixes"] = _prefixes(case)
    s["prefix"] = torch.tensor(s["prefixes"], dtype=torch.int32, device=dev) if case["prefix"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    q, k = s["q"], s["k"]
    (T, H, d), G = q.shape, case["kv_heads"]
    s["q_out"], s["k_out"] = torch.empty(T, H, d, dtype=q.dtype, device=q.device), torch.empty(T, G, d, dtype=q.dtype, device=q.device)
    if "v" in s:
        s["lse"] = torch.empty(H, T, device=q.device)
        s["dq"] = torch.empty(T, H, d, dtype=q.dtype, device=q.device)
        s["dk"], s["dv"] = (torch.empty(T, G, d, dtype=q.dtype, device=q.device) for _ in range(2))
    if own:
        from paper_2609_34420_b200 import binding as gt
        s["gt"] = gt
        single = len(s["sizes"]) == 1
        s["batch"] = gt.Batch(T, len(s["sizes"]), max(s["sizes"]), None if single else s["cu_seqlens"])
        if "v" in s:
            s["ws_fwd"] = gt._workspace(gt.gt_position_attn_fwd_workspace(s["batch"], H, G, d), q.device)
            s["ws_bwd"] = gt._workspace(gt.gt_position_attn_bwd_workspace(s["batch"], H, G, d), q.device)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _scores(q, k, i, j, case, slopes, prefix):
    """Scores [H, rows, n] of queries at positions i, their -inf where masked, and tanh(x / cap) (None without a cap)."""
    x = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(q.shape[2])
    t = None
    if case["cap"]:
        t = torch.tanh(x / case["cap"])
        x = case["cap"] * t
    if slopes is not None:
        x = x - slopes[:, None, None] * (j[None, :] - i[:, None]).abs()
    if case["causal"]:
        x = x.masked_fill((j[None, :] > i[:, None]) & (j[None, :] >= prefix), -math.inf)
    return x, t


def _plain_attn(s):
    case, q, k, v = s["case"], s["q"], s["k"], s["v"]
    T, H, d = q.shape
    G, dev, train = k.shape[1], q.device, case["what"] == "train"
    out, lse = torch.zeros(T, H, d, device=dev), torch.zeros(H, T, device=dev)
    dq, dk, dv = torch.zeros(T, H, d, device=dev), torch.zeros(T, G, d, device=dev), torch.zeros(T, G, d, device=dev)
    for a, n, prefix in zip(s["ends"], s["sizes"], s["prefixes"]):
        kk, vv = (t[a:a + n].float().repeat_interleave(H // G, 1).transpose(0, 1) for t in (k, v))
        j = torch.arange(n, device=dev)
        step = max(1, ROWS_AT_A_TIME // (H * n))
        for b in range(0, n, step):
            at = slice(a + b, a + min(n, b + step))
            qq = q[at].float().transpose(0, 1)
            x, t = _scores(qq, kk, j[b:b + step], j, case, s["slopes"], prefix)
            top = x.amax(2, keepdim=True)
            p = torch.exp(x - top)
            l = p.sum(2, keepdim=True)
            p = p / l
            o = torch.matmul(p, vv)
            out[at], lse[:, at] = o.transpose(0, 1), (top + torch.log(l))[:, :, 0]
            if train:
                do = s["dout"][at].float().transpose(0, 1)
                dv[a:a + n] += torch.matmul(p.transpose(1, 2), do).view(G, H // G, n, d).sum(1).transpose(0, 1)
                ds = p * (torch.matmul(do, vv.transpose(1, 2)) - (do * o).sum(2, keepdim=True))
                if t is not None:
                    ds = ds * (1 - t * t)
                ds = ds / math.sqrt(d)
                dq[at] = torch.matmul(ds, kk).transpose(0, 1)
                dk[a:a + n] += torch.matmul(ds.transpose(1, 2), qq).view(G, H // G, n, d).sum(1).transpose(0, 1)
    if not train:
        return out.to(q.dtype), lse
    return [out.to(q.dtype), lse] + [x.to(q.dtype) for x in (dq, dk, dv)]


def _plain_rotary(s):
    case, rot = s["case"], s["case"]["rot_dim"]
    p = s["positions"]
    if p is None:
        n = torch.tensor(s["sizes"], device=s["q"].device)
        p = torch.arange(sum(s["sizes"]), device=s["q"].device) - torch.repeat_interleave(s["cu_seqlens"][:-1], n)
    angle = p.double()[:, None] * s["frequencies"][None, :]
    sign = -1.0 if case["what"] == "inverse" else 1.0
    cos, sin = ((f(angle) * w * case["scale"]).float()[:, None, :] for f, w in ((torch.cos, 1.0), (torch.sin, sign)))
    done = []
    for x in (s["q"], s["k"]):
        y = x.float().clone()
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        y[..., a] = x[..., a].float() * cos - x[..., b].float() * sin
        y[..., b] = x[..., a].float() * sin + x[..., b].float() * cos
        done.append(y.to(x.dtype))
    return done


def run(s):
    case = s["case"]
    if not own:
        return _plain_rotary(s) if "frequencies" in s else _plain_attn(s)
    gt, q, k = s["gt"], s["q"], s["k"]
    if "frequencies" in s:
        gt.gt_rotary(q, k, s["frequencies"], s["positions"], s["batch"], case["interleaved"], case["scale"],
                     case["what"] == "inverse", s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    gt.gt_position_attn_fwd(q, k, s["v"], s["slopes"], s["prefix"], s["batch"], case["causal"], case["cap"],
                            s["q_out"], s["lse"], s["ws_fwd"])
    if case["what"] == "fwd":
        return s["q_out"], s["lse"]
    gt.gt_position_attn_bwd(q, k, s["v"], s["q_out"], s["dout"], s["lse"], s["slopes"], s["prefix"], s["batch"],
                            case["causal"], case["cap"], s["dq"], s["dk"], s["dv"], s["ws_bwd"])
    return [s[x] for x in ("q_out", "lse", "dq", "dk", "dv")]


def work(case):
    """Every tensor once in each direction; two contractions forward and five backward over the pairs that the mask leaves."""
    sizes, H, G, d = _lengths(case), case["heads"], case["kv_heads"], case["head_dim"]
    T = sum(sizes)
    if "rot_dim" in case:
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": 2 * size * T * (H + G) * d + (4 * T if case["positions"] else 0), "flops": 3 * T * (H + G) * case["rot_dim"]}
    pairs = sum(n * n - ((n * (n - 1) - p * (p - 1)) // 2 if case["causal"] else 0) for n, p in zip(sizes, _prefixes(case)))
    q, kv, rows = 2 * T * H * d, 4 * T * G * d, 4 * T * H
    fwd = {"bytes": 2 * q + kv + rows, "flops": 4 * H * d * pairs}
    if case["what"] == "fwd":
        return fwd
    return {"bytes": fwd["bytes"] + 4 * q + 2 * kv + rows, "flops": fwd["flops"] + 10 * H * d * pairs}


# ------------------------------------------------------------------------------------------ from the definition, in 64 bits
def _exact_attn(case, s):
    """Softmax rows by their log-sum-exp, gradients by automatic differentiation of the sum of out x dout."""
    T, H, d = s["q"].shape
    G, dev, train = case["kv_heads"], s["q"].device, case["what"] == "train"
    q, k, v, do = (s[x].double() for x in ("q", "k", "v", "dout"))
    out, lse = torch.zeros_like(q), torch.zeros(H, T, dtype=torch.float64, device=dev)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, n, prefix in zip(s["ends"], s["sizes"], s["prefixes"]):
        step = max(1, (1 << 26) // (n * (H // G)))
        pos = torch.arange(n, device=dev)
        for g in range(G):
            of = slice(g * (H // G), (g + 1) * (H // G))
            kk, vv = (t[a:a + n, g].clone().requires_grad_(train) for t in (k, v))
            for b in range(0, n, step):
                at = slice(a + b, a + min(n, b + step))
                qq = q[at, of].clone().requires_grad_(train)
                x = torch.einsum("ihd,jd->hij", qq, kk) * d ** -0.5
                x = torch.tanh(x / case["cap"]) * case["cap"] if case["cap"] else x
                far = (pos[b:b + step, None] - pos[None, :]).double()
                if s["slopes"] is not None:
                    x = x - s["slopes"][of].double()[:, None, None] * far.abs()
                if case["causal"]:
                    x = torch.where((far >= 0) | (pos[None, :] < prefix), x, -math.inf)
                m = torch.logsumexp(x, 2)
                o = torch.einsum("hij,jd->ihd", torch.exp(x - m[:, :, None]), vv)
                out[at, of], lse[of, at] = o.detach(), m.detach()
                if train:
                    (o * do[at, of]).sum().backward()
                    dq[at, of] = qq.grad
            if train:
                dk[a:a + n, g], dv[a:a + n, g] = kk.grad, vv.grad
    return [out, lse, dq, dk, dv] if train else (out, lse)


def _exact_rotary(case, s):
    """Pairs of channels as complex numbers, times scale e^(i angle)."""
    rot, dev = case["rot_dim"], s["q"].device
    p = torch.cat([torch.arange(n, dtype=torch.float64, device=dev) for n in s["sizes"]])
    p = p if s["positions"] is None else s["positions"].double()
    i = torch.arange(rot // 2, dtype=torch.float64, device=dev)
    angle = torch.outer(p, 10000.0 ** (-2 * i / rot)) * (-1 if case["what"] == "inverse" else 1)
    turn = torch.polar(torch.full_like(angle, case["scale"]), angle)[:, None, :]
    done = []
    for x in (s["q"].double(), s["k"].double()):
        r = x[..., :rot]
        pairs = r.unflatten(2, (-1, 2)) if case["interleaved"] else r.unflatten(2, (2, -1)).transpose(2, 3)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        z = z.flatten(2) if case["interleaved"] else z.transpose(2, 3).flatten(2)
        done.append(torch.cat([z, x[..., rot:]], 2))
    return done


def exact(case, seed):
    s = _inputs(case, seed)
    return _exact_rotary(case, s) if "rot_dim" in case else _exact_attn(case, s)
