"""The operators at the entry of the stage behind the encoder -- embeddings of texts and visual tokens, the norm that adds to the
residual stream, rows in 8 bits, products of such rows -- as cases for timing and checking them.

Six kinds, each one pass as a program makes it:

  embed       rows of sequences of text and visual tokens                 (``Embedding.forward``)
  embed_grad  gradients of the table and of the visual rows, given dout   (``Embedding.backward``)
  norm        x + residual and its RMS norm, in its own type or in 8 bits and read back
              (``AddNorm.forward``, ``dequant_rows``)
  norm_train  the same and every gradient, given dy and dsum              (``AddNorm.forward``, ``backward``)
  quant       rows to 8 bits with a scale each, and back                  (``quant_rows``, ``dequant_rows``)
  linear      product of 8-bit rows and 8-bit weights                     (``Int8Linear.forward``)

Where ``own`` is false the operators are computed in their plain form: elementary torch operations in fp32.
"""

import math

import torch

own = False

DEVICE = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEAST = 2.0 ** -100          # largest magnitude that a row in 8 bits is taken to have at least
EPS = 1e-6
NO_ROW = 2 ** 31 - 1         # an id of no row: padding


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one new token for each of 32 chats, into an fp32 residual stream: latency
        {"name": "embed-decode", "kind": "embed", "dtype": "bf16", "out": "f32", "tokens": 32, "vocab": 131072, "hidden": 3200, "visual": 0, "pad": 0.0, "hot": 0.1, "scale": 1.0},
        # a prompt of text around the visual tokens of four clips
        {"name": "embed-prompt", "kind": "embed", "dtype": "bf16", "out": "bf16", "tokens": 16384, "vocab": 131072, "hidden": 3584, "visual": 8192, "pad": 0.0, "hot": 0.1, "scale": 59.866519},
        # training step of one chat with an image: few tokens, a small table
        {"name": "embed-grad-chat", "kind": "embed_grad", "dtype": "bf16", "out": "bf16", "tokens": 2049, "vocab": 32000, "hidden": 1024, "visual": 256, "pad": 0.0, "hot": 0.1, "scale": 32.0},
        # training step of a padded batch: a large table, a token that takes every fifth place
        {"name": "embed-grad-batch", "kind": "embed_grad", "dtype": "bf16", "out": "f32", "tokens": 32768, "vocab": 131072, "hidden": 3200, "visual": 8192, "pad": 0.1, "hot": 0.2, "scale": 1.0},
        # one new token for each of 16 chats: latency
        {"name": "norm-decode", "kind": "norm", "dtype": "bf16", "residual": "f32", "tokens": 16, "hidden": 3200, "quant": False},
        # the patch tokens of four clips, for a product in 8 bits
        {"name": "norm-4-clips", "kind": "norm", "dtype": "bf16", "residual": "f32", "tokens": 32768, "hidden": 3200, "quant": True},
        # training step on eight 448 x 448 images
        {"name": "norm-train-8-images", "kind": "norm_train", "dtype": "bf16", "residual": "bf16", "tokens": 6272, "hidden": 1024},
        # the weights of a 3200 / 12 800 block when they are loaded
        {"name": "quant-weights", "kind": "quant", "dtype": "bf16", "rows": 12800, "cols": 3200},
        # fp32 rows of an odd length, one 2688 x 2688 image after the 2 x 2 merge and one more
        {"name": "quant-odd", "kind": "quant", "dtype": "f32", "rows": 7057, "cols": 1153},
        # one token of one chat through a 3200 / 12 800 linear: the weights' way to the chip
        {"name": "linear-1-token", "kind": "linear", "out": "bf16", "tokens": 1, "hidden": 3200, "width": 12800, "bias": False},
        # one 2688 x 2688 image after the merge and one more row, a width that no tile divides
        {"name": "linear-image", "kind": "linear", "out": "bf16", "tokens": 7057, "hidden": 1152, "width": 4304, "bias": True},
        # the four clips of the video encoder: the largest pass
        {"name": "linear-4-clips", "kind": "linear", "out": "bf16", "tokens": 32768, "hidden": 3200, "width": 12800, "bias": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_train", "quant", "linear", "linear", "linear"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    wide = "f32" if dtype == "f32" else rng.choice(["bf16", "f32"])      # outputs and residual streams are at least as wide
    if kind in ("embed", "embed_grad"):
        D = rng.choice([1024, 1152, 3200, 3584, 0, 0, 0])
        D = D or _log_int(rng, 1, 4096)
        V = _log_int(rng, 100, 131072)
        T = _log_int(rng, 1, int(min(32768, 1.2e8 / D)))
        R = rng.choice([0, rng.randint(0, T)])
        return {"kind": kind, "dtype": dtype, "out": wide, "tokens": T, "vocab": V, "hidden": D, "visual": R, "pad": rng.choice([0.0, 0.1, 0.5]),
                "hot": rng.choice([0.0, 0.1, 0.9]), "scale": rng.choice([1.0, math.sqrt(D)])}
    if kind in ("norm", "norm_train"):
        D = rng.choice([1024, 1152, 3200, 3584, 0, 0, 0])
        D = D or _log_int(rng, 1, 16384)
        T = _log_int(rng, 1, int(min(32768, 1.2e8 / D)))
        c = {"kind": kind, "dtype": dtype, "residual": wide, "tokens": T, "hidden": D}
        return {**c, "quant": rng.random() < 0.5} if kind == "norm" else c
    if kind == "quant":
        cols = _log_int(rng, 1, 16384)
        return {"kind": kind, "dtype": dtype, "rows": _log_int(rng, 1, int(min(32768, 1.2e8 / cols))), "cols": cols}
    K, N = rng.choice([(1024, 4096), (4096, 1024), (1152, 4304), (3200, 12800), (12800, 3200), (3200, 9600), (0, 0), (0, 0), (0, 0)])
    if K == 0:
        K, N = 16 * _log_int(rng, 2, 640), 8 * _log_int(rng, 2, 1280)
    most = min(32768, 2.6e12 / (2.0 * K * N))
    return {"kind": kind, "out": rng.choice(["bf16", "bf16", "f32"]), "tokens": _log_int(rng, 1, max(64, int(most))), "hidden": K, "width": N, "bias": rng.random() < 0.5}


# ------------------------------------------------------------------ what a program has in hand

def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    s, kind = dict(case), case["kind"]

    def randn(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).mul_(std).to(dtype)

    def rand(n):
        return torch.rand(n, generator=gen, device=DEVICE)

    if kind in ("embed", "embed_grad"):
        T, V, D, R, dt = case["tokens"], case["vocab"], case["hidden"], case["visual"], DTYPES[case["dtype"]]
        ids = (V * rand(T).double() ** 3).long().clamp(max=V - 1)               # low ids are frequent
        ids = torch.where(rand(T) < case["hot"], torch.full_like(ids, V // 7), ids)
        at = int(torch.randint(0, T - R + 1, (1,), generator=gen, device=DEVICE).item())
        ids[at:at + R] = -1 - torch.arange(R, device=DEVICE)                    # the visual tokens, in one piece
        s["ids"] = torch.where(rand(T) < case["pad"], torch.full_like(ids, NO_ROW), ids).to(torch.int32)
        if kind == "embed":
            s["table"] = randn(V, D, std=0.02, dtype=dt)
            s["visual_rows"] = randn(R, D, dtype=dt) if R else None
        else:
            s["dout"] = randn(T, D, dtype=DTYPES[case["out"]])
        if own:
            from paper_2601_11590_amd import binding as B
            s["op"] = B.Embedding(case["dtype"], V, D, out=case["out"], scale=case["scale"], max_tokens=T, training=kind == "embed_grad")
    elif kind in ("norm", "norm_train"):
        T, D, dt, rt = case["tokens"], case["hidden"], DTYPES[case["dtype"]], DTYPES[case["residual"]]
        s["x"], s["r"], s["gain"] = randn(T, D, dtype=dt), randn(T, D, std=3.0, dtype=rt), (1.0 + randn(D, std=0.1)).to(dt)
        if kind == "norm_train":
            s["dy"], s["dsum"] = randn(T, D, dtype=dt), randn(T, D, dtype=rt)
        if own:
            from paper_2601_11590_amd import binding as B
            s["op"] = B.AddNorm(case["dtype"], D, residual=case["residual"], eps=EPS, max_tokens=T, training=kind == "norm_train")
    elif kind == "quant":
        s["x"] = randn(case["rows"], case["cols"], std=0.02, dtype=DTYPES[case["dtype"]])
    else:
        T, K, N = case["tokens"], case["hidden"], case["width"]

        def held(rows, std):                                                    # rows of normal values as 8 bits hold them
            scale = (std * 4.2 / 127.0) * (0.8 + 0.4 * rand(rows))
            return (randn(rows, K, std=std).div_(scale[:, None])).round_().clamp_(-127, 127).to(torch.int8), scale
        s["x"], s["x_scale"] = held(T, 1.0)
        w, w_scale = held(N, 0.02)
        s["w"] = {"w": w, "scale": w_scale}
        if case["bias"]:
            s["w"]["bias"] = randn(N, std=0.02)
        if own:
            from paper_2601_11590_amd import binding as B
            s["op"] = B.Int8Linear(K, N, out=case["out"], max_tokens=T, use_bias=case["bias"])
    return s


# ------------------------------------------------------------------ one pass, plain

def _embed(s):
    ids, V = s["ids"].long(), s["vocab"]
    out = s["table"][ids.clamp(0, V - 1)].float() * s["scale"] * ((ids >= 0) & (ids < V))[:, None]
    if s["visual"]:
        out = torch.where((ids < 0)[:, None], s["visual_rows"][(-1 - ids).clamp(0, s["visual"] - 1)].float(), out)
    return out.to(DTYPES[s["out"]])


def _embed_grad(s):
    ids, V, R, D, dt = s["ids"].long(), s["vocab"], s["visual"], s["hidden"], DTYPES[s["dtype"]]
    d = s["dout"].float()
    row = torch.where(ids < 0, V - 1 - ids, torch.where(ids < V, ids, V + R))   # table, visual rows, and one for those of none
    sums = torch.zeros(V + R + 1, D, device=DEVICE).index_add_(0, row, d)
    out = {"table": (sums[:V] * s["scale"]).to(dt)}
    if R:
        out["rows"] = sums[V:V + R].to(dt)
    return out


def _norm(s):
    h = s["x"].float() + s["r"].float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS) * s["gain"].float()
    return h, y


def _eight_bits(v):
    most = v.abs().amax(dim=1, keepdim=True).clamp(min=LEAST)
    scale = most * (1.0 / 127.0)
    return torch.round(v * (torch.full_like(most, 127.0) / most)) * scale, scale[:, 0]


def _norm_train(s):
    h, y = _norm(s)
    dt, rt = DTYPES[s["dtype"]], DTYPES[s["residual"]]
    kept = h.to(rt).float()                        # the gradients are those at the sum as it is kept
    r = torch.rsqrt(kept.square().mean(dim=1, keepdim=True) + EPS)
    n, dy = kept * r, s["dy"].float()
    g = dy * s["gain"].float()
    dx = s["dsum"].float() + r * (g - n * (g * n).mean(dim=1, keepdim=True))
    out = {"sum": h.to(rt), "y": y.to(dt), "dx": dx.to(dt), "gain": (dy * n).sum(dim=0).to(dt)}
    return out if dt == rt else {**out, "dresidual": dx.to(rt)}


def _linear(s):
    y = s["x"].float() @ s["w"]["w"].float().t() * s["x_scale"][:, None] * s["w"]["scale"]
    if s["bias"]:
        y = y + s["w"]["bias"]
    return y.to(DTYPES[s["out"]])


# ------------------------------------------------------------------ one pass

def run(state):
    s, kind = state, state["kind"]
    if kind == "embed":
        return s["op"].forward(s["table"], s["ids"], s["visual_rows"]) if own else _embed(s)
    if kind == "embed_grad":
        return s["op"].backward(s["ids"], s["dout"], num_rows=s["visual"]) if own else _embed_grad(s)
    if kind == "norm":
        if own:
            from paper_2601_11590_amd import binding as B
            if not s["quant"]:
                return s["op"].forward(s["gain"], s["x"], s["r"], want=("sum", "y"))
            o = s["op"].forward(s["gain"], s["x"], s["r"], want=("sum", "q"))
            return {"sum": o["sum"], "values": B.dequant_rows(o["q"], o["scale"], "bf16"), "scale": o["scale"]}
        h, y = _norm(s)
        h = h.to(DTYPES[s["residual"]])
        if not s["quant"]:
            return {"sum": h, "y": y.to(DTYPES[s["dtype"]])}
        values, scale = _eight_bits(y)
        return {"sum": h, "values": values.to(torch.bfloat16), "scale": scale}
    if kind == "norm_train":
        if not own:
            return _norm_train(s)
        o = s["op"].forward(s["gain"], s["x"], s["r"], want=("sum", "y"))
        want = ("dx", "gain") if s["dtype"] == s["residual"] else ("dx", "dresidual", "gain")
        return {**o, **s["op"].backward(s["gain"], o["sum"], s["dy"], dsum=s["dsum"], want=want)}
    if kind == "quant":
        if own:
            from paper_2601_11590_amd import binding as B
            q, scale = B.quant_rows(s["x"])
            return {"values": B.dequant_rows(q, scale, "bf16"), "scale": scale}
        values, scale = _eight_bits(s["x"].float())
        return {"values": values.to(torch.bfloat16), "scale": scale}
    return s["op"].forward(s["w"], s["x"], s["x_scale"]) if own else _linear(s)


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "embed":
        every = s["table"].double() * case["scale"]
        if case["visual"]:
            every = torch.cat([s["visual_rows"].double().flip(0), every])      # id -1 - j is j rows ahead of row 0
        every = torch.cat([every, every.new_zeros(1, case["hidden"])])
        return every[(s["ids"].long() + case["visual"]).clamp(max=len(every) - 1)]
    if kind == "embed_grad":
        V, R, d = case["vocab"], case["visual"], s["dout"].double()
        out = {"table": torch.zeros(V, case["hidden"], dtype=torch.float64, device=DEVICE)}
        text = ((s["ids"] >= 0) & (s["ids"] < V)).nonzero()[:, 0]
        out["table"].index_put_((s["ids"][text].long(),), d[text] * case["scale"], accumulate=True)
        if R:
            seen = (s["ids"] < 0).nonzero()[:, 0]
            out["rows"] = torch.zeros(R, case["hidden"], dtype=torch.float64, device=DEVICE)
            out["rows"].index_put_((-1 - s["ids"][seen].long(),), d[seen], accumulate=True)
        return out
    if kind == "quant":
        v = s["x"].double()
        most = v.abs().amax(dim=1).clamp(min=LEAST)
        return {"values": (v / (most / 127)[:, None]).round() * (most / 127)[:, None], "scale": most / 127}
    if kind == "linear":
        y = torch.nn.functional.linear(s["x"].double() * s["x_scale"].double()[:, None], s["w"]["w"].double() * s["w"]["scale"].double()[:, None])
        return y + s["w"]["bias"].double() if case["bias"] else y
    h, gain = s["x"].double() + s["r"].double(), s["gain"].double()
    y = h / (h.pow(2).sum(dim=1, keepdim=True) / case["hidden"] + EPS).sqrt() * gain
    if kind == "norm" and case["quant"]:
        step = y.abs().amax(dim=1, keepdim=True).clamp(min=LEAST) / 127
        return {"sum": h, "values": (y / step).round() * step, "scale": step[:, 0]}
    if kind == "norm":
        return {"sum": h, "y": y}
    kept, gain = h.to(DTYPES[case["residual"]]).double().requires_grad_(), gain.requires_grad_()
    n = kept / (kept.pow(2).sum(dim=1, keepdim=True) / case["hidden"] + EPS).sqrt()
    dx, dgain = torch.autograd.grad((n * gain * s["dy"].double()).sum() + (kept * s["dsum"].double()).sum(), (kept, gain))
    out = {"sum": h, "y": y.detach(), "dx": dx, "gain": dgain}
    return out if case["dtype"] == case["residual"] else {**out, "dresidual": dx}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    size, kind = {"f32": 4.0, "bf16": 2.0}, case["kind"]
    if kind in ("embed", "embed_grad"):
        T, V, R, D, es, os = case["tokens"], case["vocab"], case["visual"], case["hidden"], size[case["dtype"]], size[case["out"]]
        if kind == "embed":
            return {"bytes": 4.0 * T + (min(T - R, V) + R) * D * es + T * D * os, "flops": 1.0 * T * D}
        return {"bytes": 4.0 * T + T * D * os + (V + R) * D * es, "flops": 1.0 * T * D}
    if kind in ("norm", "norm_train"):
        T, D, es, rs = case["tokens"], case["hidden"], size[case["dtype"]], size[case["residual"]]
        if kind == "norm_train":
            return {"bytes": T * D * (4 * es + 3 * rs + (0 if es == rs else rs)) + 2 * D * es, "flops": 17.0 * T * D}
        if case["quant"]:                         # the values in 8 bits, and read back
            return {"bytes": T * D * (es + 2 * rs + 3.0) + 4.0 * T + D * es, "flops": 8.0 * T * D}
        return {"bytes": T * D * (2 * es + 2 * rs) + D * es, "flops": 5.0 * T * D}
    if kind == "quant":
        return {"bytes": case["rows"] * (case["cols"] * (size[case["dtype"]] + 3.0) + 4.0), "flops": 4.0 * case["rows"] * case["cols"]}
    T, K, N = case["tokens"], case["hidden"], case["width"]
    return {"bytes": 1.0 * (T + N) * K + 4.0 * (T + N) + T * N * size[case["out"]] + (4.0 * N if case["bias"] else 0.0), "flops": 2.0 * T * K * N}
