"""Layer norm, rotary positions with several axes, and sliding-window attention
over packed sequences: the calls whose speed counts, their plain forms and
their definitions in 64 bits.

Each case is one pass through one operator of the library, as a training
program calls it:

  layernorm  rows normalised to mean 0 and variance 1, gain and bias; `train`
             is the forward and then the backward pass with both weight
             gradients
  rope       rotary positions over up to four axes (time, height, width) of
             packed head rows: rotated forward, rotated back (`backward`), or
             the cos/sin table that the projection's epilogue takes (`table`)
  attention  causal attention over packed sequences, in which a token sees
             the last `window` tokens of its sequence and the sequence's first
             `sinks`; `train` is the forward and then the backward pass
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False  # True: run() makes the library's calls; False: the plain forms

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5


def _norm(name, direction, tokens, d, x, w, y, dy="fp32", residual=False):
    c = {"op": "layernorm", "pass": direction, "tokens": tokens, "d": d, "x": x, "w": w, "y": y,
         "dy": dy, "residual": residual}
    return {"name": name, **c} if name else c


def _rope(name, direction, tokens, heads, hd, dtype, sections, freq, base, reach):
    c = {"op": "rope", "pass": direction, "tokens": tokens, "heads": heads, "hd": hd,
         "dtype": dtype, "sections": sections, "freq": freq, "base": base, "reach": reach}
    return {"name": name, **c} if name else c


def _attn(name, direction, dtype, tokens, seqs, tail, heads, kv, hd, window, sinks, split):
    c = {"op": "attention", "pass": direction, "dtype": dtype, "tokens": tokens, "seqs": seqs,
         "tail": tail, "heads": heads, "kv": kv, "hd": hd, "window": window, "sinks": sinks,
         "split": split}
    return {"name": name, **c} if name else c


def listed():
    return [
        # a few tokens through a small model: the call's latency
        _norm("layernorm_t9_d768", "forward", 9, 768, "fp32", "fp32", "fp32"),
        # a 7B-shaped layer's microbatch: fp32 residual stream in, bf16 operand out, the
        # residual's gradient added on the way back
        _norm("layernorm_train_t4096_d4096", "train", 4096, 4096, "fp32", "bf16", "bf16", "fp32", True),
        # ragged rows of an odd width, everything in 16 bits
        _norm("layernorm_train_t3001_d1155", "train", 3001, 1155, "bf16", "bf16", "bf16", "bf16", False),
        # a long packed microbatch of a wide model
        _norm("layernorm_train_t16411_d8192", "train", 16411, 8192, "bf16", "fp32", "bf16", "bf16", True),
        # one image and a question behind it: q and k rows of 32 and 8 heads, three axes
        _rope("rope_image_t1601", "forward", 1601, 40, 128, "bf16", "16,24,24", "head", 1000000.0, 1200),
        # the gradient of a video's q and k rows, every axis with frequencies of its own,
        # the last pairs of a head without position
        _rope("rope_video_back_t32760", "backward", 32760, 24, 128, "bf16", "22,20,20", "axis", 10000.0, 2048),
        # cos and sin of a long mixed document, positions far from 0
        _rope("rope_table_t8192", "table", 8192, 1, 128, "fp32", "16,24,24", "head", 500000.0, 1048576),
        # a handful of short sequences through a small model: the call's latency
        _attn("attention_t77", "forward", "bf16", 77, 5, 3, 8, 8, 64, 32, 2, 11),
        # a 7B-shaped layer's microbatch with a window of a quarter of its length
        _attn("attention_train_t4096", "train", "bf16", 4096, 1, 0, 32, 32, 128, 1024, 4, 0),
        # packed documents of unequal length, grouped-query attention, fp16 q, k and v as the
        # projections leave them, a padded end
        _attn("attention_train_gqa_t8100", "train", "fp16", 8100, 9, 37, 32, 8, 128, 512, 16, 5),
        # one long document, grouped-query attention
        _attn("attention_train_t32768", "train", "bf16", 32768, 1, 0, 16, 4, 128, 4096, 64, 0),
        # a small model in full precision, packed
        _attn("attention_train_fp32_t600", "train", "fp32", 600, 4, 0, 12, 12, 64, 128, 4, 7),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _divisor(rng, n):
    return rng.choice([k for k in range(1, n + 1) if n % k == 0])


def draw(rng):
    op = rng.choice(["layernorm", "layernorm", "rope", "rope", "attention", "attention", "attention"])
    top = max(work(c)["bytes"] if op != "attention" else work(c)["flops"]
              for c in listed() if c["op"] == op)
    while True:
        if op == "layernorm":
            d = round(_log(rng, 64, 12288))
            if rng.random() < 0.7:
                d = max(64, 8 * round(d / 8))
            x = rng.choice(["fp32", "bf16", "fp16"])
            c = _norm("", rng.choice(["forward", "train", "train"]), round(_log(rng, 1, 32768)), d,
                      x, rng.choice(["fp32", "bf16"]), rng.choice(["fp32", "bf16"] if x == "fp32" else [x]),
                      rng.choice(["fp32", "bf16"]), rng.random() < 0.5)
        elif op == "rope":
            hd = rng.choice([32, 64, 72, 80, 96, 128, 128, 128])
            half, n = hd // 2, rng.randint(1, 4)
            first = half // (2 * n) if n > 1 else half
            rest = (half - first) // (n - 1) if n > 1 else 0
            if rng.random() < 0.3 and rest > 1:
                rest -= 1  # some pairs without position
            c = _rope("", rng.choice(["forward", "backward", "table"]), round(_log(rng, 1, 32768)),
                      rng.randint(1, 48), hd, rng.choice(["fp32", "bf16", "fp16"]),
                      ",".join(str(k) for k in [first] + [rest] * (n - 1)), rng.choice(["head", "axis"]),
                      rng.choice([10000.0, 500000.0, 1000000.0]), round(_log(rng, 16, 1 << 20)))
        else:
            dtype = rng.choice(["bf16", "bf16", "bf16", "fp16", "fp32"])
            full = dtype == "fp32"
            heads = round(_log(rng, 1, 12 if full else 40))
            tokens = round(_log(rng, 16, 2000 if full else 32768))
            seqs = min(round(_log(rng, 1, 24)), tokens // 8)
            c = _attn("", rng.choice(["forward", "train", "train"]), dtype, tokens, seqs,
                      rng.choice([0, 0, rng.randint(1, 70)]), heads,
                      _divisor(rng, heads) if rng.random() < 0.6 else heads,
                      rng.choice([16, 32, 48, 64, 80, 128]) if full else rng.choice([64, 128, 128]),
                      round(_log(rng, 8, 4096)), rng.choice([0, 1, 4, rng.randint(2, 128)]),
                      rng.randint(1, 1 << 20))
        if op != "attention":
            fits = work(c)["bytes"] <= top
        else:  # (the plain form's scores and gathered sinks are bounded too)
            fits = work(c)["flops"] <= (5e10 if c["dtype"] == "fp32" else top) and \
                c["tokens"] * c["heads"] * (min(1024, c["window"]) + c["window"]) <= 2.7e9 and \
                c["tokens"] * c["kv"] * c["hd"] * c["sinks"] <= 1.1e9
        if fits:
            return c


# ------------------------------------------------------------------ sizes

def _lengths(c):
    """Lengths of the packed sequences: `tokens` cut at random places into `seqs` parts of two
    tokens at least."""
    n, s = c["tokens"], c["seqs"]
    cuts = sorted(random.Random(c["split"]).choices(range(n - 2 * s + 1), k=s - 1))
    ends = [x + 2 * (i + 1) for i, x in enumerate(cuts)] + [n]
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def _pairs(c):
    """Query-key pairs that attention visits, per head."""
    total = 0
    for n in _lengths(c):
        seen = np.arange(1, n + 1, dtype=np.int64)
        total += int((np.minimum(seen, c["window"]) +
                      np.minimum(c["sinks"], np.maximum(seen - c["window"], 0))).sum())
    return total


def work(case):
    c = case
    if c["op"] == "layernorm":
        n, d = c["tokens"] * c["d"], c["d"]
        b, f = n * (SIZE[c["x"]] + SIZE[c["y"]]) + 8 * c["tokens"] + 2 * d * SIZE[c["w"]], 8 * n
        if c["pass"] == "train":  # x, dy (and the residual's gradient) in, dx out, dg, db
            b += n * (2 * SIZE[c["x"]] + SIZE[c["dy"]]) + 8 * c["tokens"] + d * (SIZE[c["w"]] + 8)
            b += n * SIZE[c["x"]] if c["residual"] else 0
            f += 14 * n
        return {"bytes": b, "flops": f}
    if c["op"] == "rope":
        axes = len(c["sections"].split(","))
        pos = 4 * axes * c["tokens"]
        if c["pass"] == "table":
            return {"bytes": pos + 4 * c["tokens"] * c["hd"], "flops": 2 * c["tokens"] * c["hd"]}
        n = c["tokens"] * c["heads"] * c["hd"]
        return {"bytes": pos + 2 * n * SIZE[c["dtype"]], "flops": 3 * n}
    T, e = c["tokens"], SIZE[c["dtype"]]
    qo, kv = T * c["heads"] * c["hd"], T * c["kv"] * c["hd"]
    o = 4 if c["dtype"] == "fp32" else 2  # o and every gradient
    b = (qo + 2 * kv) * e + qo * o + 4 * T * c["heads"]
    f = 4 * _pairs(c) * c["heads"] * c["hd"]
    if c["pass"] == "train":  # q, k, v, o, lse and dout in, dq, dk, dv out; five products
        b += (qo + 2 * kv) * (e + o) + 2 * qo * o + 4 * T * c["heads"]
        f += 10 * _pairs(c) * c["heads"] * c["hd"]
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


def prepare(case, seed):
    """The operator's inputs, and the output buffers that the program keeps."""
    c, g, s = case, _gen(seed), {"case": case}
    if c["op"] == "layernorm":
        T, d = c["tokens"], c["d"]
        x = _randn(g, (T, d), 1.0, torch.float32)
        x += torch.randn(T, 1, generator=g, device=DEV) * 0.5  # rows off 0
        x *= torch.exp(torch.randn(d, generator=g, device=DEV) * 0.5)  # channels of unequal size
        s["x"] = x.to(DTYPES[c["x"]])
        s["g"] = _randn(g, d, 0.1, torch.float32).add_(1.0).to(DTYPES[c["w"]])
        s["b"] = _randn(g, d, 0.1, DTYPES[c["w"]])
        s["y"] = torch.empty((T, d), dtype=DTYPES[c["y"]], device=DEV)
        s["mean"], s["rstd"] = (torch.empty(T, device=DEV) for _ in range(2))
        if c["pass"] == "train":
            s["dy"] = _randn(g, (T, d), 0.5, DTYPES[c["dy"]])
            s["dres"] = _randn(g, (T, d), 0.5, DTYPES[c["x"]]) if c["residual"] else None
            s["dx"] = torch.empty_like(s["x"])
            s["dg"], s["db"] = (torch.empty(d, device=DEV) for _ in range(2))
    elif c["op"] == "rope":
        T, axes, hd = c["tokens"], len(c["sections"].split(",")), c["hd"]
        # the first axis grows along the tokens, the others walk a grid of it
        first = torch.arange(T, device=DEV, dtype=torch.int32) % c["reach"]
        first += int(torch.randint(0, max(1, c["reach"] - T), (1,), generator=g, device=DEV))
        rest = torch.randint(0, c["reach"], (axes - 1, T), generator=g, device=DEV, dtype=torch.int32)
        s["pos"] = torch.cat([first[None], rest]).contiguous()
        if c["pass"] == "table":
            s["cos"], s["sin"] = (torch.empty((T, hd // 2), device=DEV) for _ in range(2))
        else:
            s["x"] = _randn(g, (T, c["heads"] * hd), 1.0, DTYPES[c["dtype"]])
            s["y"] = torch.empty_like(s["x"])
    else:
        rows, H, kv, hd = c["tokens"] + c["tail"], c["heads"], c["kv"], c["hd"]
        dt, out = DTYPES[c["dtype"]], torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
        s["qkv"] = _randn(g, (rows, (H + 2 * kv) * hd), 1.0, dt)
        s["dout"] = _randn(g, (rows, H * hd), 0.25, out)
        ends = np.cumsum([0] + _lengths(c)).astype(np.int32)
        s["offsets"] = torch.from_numpy(ends).to(DEV)
        # the rows behind the last sequence stay as they are
        s["o"] = torch.zeros((rows, H * hd), dtype=out, device=DEV)
        s["lse"] = torch.zeros((H, rows), device=DEV)
        if c["pass"] == "train":
            s["dqkv"] = torch.zeros((rows, (H + 2 * kv) * hd), dtype=out, device=DEV)
    return s


# ------------------------------------------------------------------ the pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"layernorm": _layernorm_own, "rope": _rope_own, "attention": _attention_own}[op](state)
    return {"layernorm": _layernorm_plain, "rope": _rope_plain, "attention": _attention_plain}[op](state)


def _scratch(s, size):
    """The workspace that the program keeps for this call (made on its first one)."""
    if "scratch" not in s:
        s["scratch_bytes"] = size()
        s["scratch"] = torch.empty(max(1, s["scratch_bytes"]), dtype=torch.uint8, device=DEV)
    return s["scratch"], s["scratch_bytes"]


def _layernorm_own(s):
    from paper_2606_11169_amd import libchunk as lc
    c = s["case"]
    code = {"fp32": lc.LC_FP32, "bf16": lc.LC_BF16, "fp16": lc.LC_FP16}
    T, d, st = c["tokens"], c["d"], torch.cuda.current_stream()
    x, w, y, dy = code[c["x"]], code[c["w"]], code[c["y"]], code[c["dy"]]
    lc.lc_layernorm_forward(T, d, s["x"], s["g"], s["b"], EPS, s["y"], s["mean"], s["rstd"], x, w, y,
                            stream=st)
    if c["pass"] == "forward":
        return {k: s[k] for k in ("y", "mean", "rstd")}
    scratch, n = _scratch(s, lambda: lc.lc_layernorm_scratch_bytes(T, d))
    lc.lc_layernorm_backward(T, d, s["dy"], s["x"], s["mean"], s["rstd"], s["g"], s["dres"], s["dx"],
                             s["dg"], s["db"], scratch, n, dy, x, w, x, x, store_dg=1, stream=st)
    return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dg", "db")}


def _rope_own(s):
    from paper_2606_11169_amd import libchunk as lc
    c, st = s["case"], torch.cuda.current_stream()
    code = {"fp32": lc.LC_FP32, "bf16": lc.LC_BF16, "fp16": lc.LC_FP16}[c["dtype"]]
    sections = [int(k) for k in c["sections"].split(",")]
    freq = lc.LC_ROPE_FREQ_AXIS if c["freq"] == "axis" else lc.LC_ROPE_FREQ_HEAD
    T = c["tokens"]
    if c["pass"] == "table":
        lc.lc_rope_axes_table(T, c["hd"], sections, s["pos"], T, s["cos"], s["sin"], base=c["base"],
                              freq=freq, stream=st)
        return {"cos": s["cos"], "sin": s["sin"]}
    call = lc.lc_rope_axes_forward if c["pass"] == "forward" else lc.lc_rope_axes_backward
    width = c["heads"] * c["hd"]
    call(T, c["heads"], c["hd"], sections, s["pos"], T, s["x"], width, s["y"], width, code, code,
         base=c["base"], freq=freq, stream=st)
    return {"y": s["y"]}


def _attention_own(s):
    from paper_2606_11169_amd import libchunk as lc
    c, st = s["case"], torch.cuda.current_stream()
    code = {"fp32": lc.LC_FP32, "bf16": lc.LC_BF16, "fp16": lc.LC_FP16}[c["dtype"]]
    out = lc.LC_FP32 if c["dtype"] == "fp32" else lc.LC_BF16
    rows, B, H, kv, hd = c["tokens"] + c["tail"], c["seqs"], c["heads"], c["kv"], c["hd"]
    ld, k0, v0 = (H + 2 * kv) * hd, H * hd, (H + kv) * hd
    x, d = s["qkv"], s.get("dqkv")
    lc.lc_window_attention_forward(code, out, rows, B, s["offsets"], H, kv, hd, c["window"], c["sinks"],
                                   x, ld, x[:, k0:], ld, x[:, v0:], ld, s["o"], H * hd, s["lse"],
                                   stream=st)
    if c["pass"] == "forward":
        return {"o": s["o"], "lse": s["lse"]}
    scratch, n = _scratch(s, lambda: lc.lc_window_attention_scratch_bytes(code, rows, H, kv, hd,
                                                                          c["window"], c["sinks"]))
    lc.lc_window_attention_backward(code, out, rows, B, s["offsets"], H, kv, hd, c["window"], c["sinks"],
                                    x, ld, x[:, k0:], ld, x[:, v0:], ld, s["o"], H * hd, s["lse"],
                                    s["dout"], H * hd, d, ld, d[:, k0:], ld, d[:, v0:], ld, scratch, n,
                                    stream=st)
    return {"o": s["o"], "lse": s["lse"], "dqkv": d}


# ------------------------------------------------------------------ plain forms

def _layernorm_plain(s):
    c = s["case"]
    x, g, b = s["x"].float(), s["g"].float(), s["b"].float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + EPS)
    xh = xc * rstd
    out = {"y": (xh * g + b).to(DTYPES[c["y"]]), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if c["pass"] == "train":
        dy = s["dy"].float()
        dxh = dy * g
        dx = rstd * (dxh - dxh.mean(1, keepdim=True) - xh * (dxh * xh).mean(1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        out |= {"dx": dx.to(s["x"].dtype), "dg": (dy * xh).sum(0), "db": dy.sum(0)}
    return out


def _angles(c, pos):
    """cos and sin of every token's pairs; the angles in 64 bits, as far positions need them."""
    sections = torch.tensor([int(k) for k in c["sections"].split(",")], device=DEV)
    half, used = c["hd"] // 2, int(sections.sum())
    axis = torch.repeat_interleave(torch.arange(len(sections), device=DEV), sections)
    pair = torch.arange(used, device=DEV, dtype=torch.float64)
    if c["freq"] == "axis":
        part = (pair - (torch.cumsum(sections, 0) - sections)[axis]) / sections[axis]
    else:
        part = pair / half
    angle = torch.zeros((pos.shape[1], half), dtype=torch.float64, device=DEV)
    angle[:, :used] = pos.double()[axis].T * c["base"] ** -part
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rope_plain(s):
    c = s["case"]
    cos, sin = _angles(c, s["pos"])
    if c["pass"] == "table":
        return {"cos": cos, "sin": sin}
    if c["pass"] == "backward":
        sin = -sin
    x = s["x"].float().view(c["tokens"], c["heads"], 2, c["hd"] // 2)
    a, b, cos, sin = x[:, :, 0], x[:, :, 1], cos[:, None], sin[:, None]
    y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=2)
    return {"y": y.to(s["x"].dtype).view(s["x"].shape)}


def _attention_plain(s):
    """Blocks of C queries against the C + W keys that end with the block, and each query's
    sinks beside them."""
    c = s["case"]
    n, H, kv, hd, W, S = c["tokens"], c["heads"], c["kv"], c["hd"], c["window"], c["sinks"]
    G, scale, rows = H // kv, 1.0 / math.sqrt(hd), c["tokens"] + c["tail"]
    C = max(64, min(1024, W))
    nb = -(-n // C)
    off = s["offsets"].long()
    start = torch.repeat_interleave(off[:-1], off[1:] - off[:-1], output_size=n)
    x = s["qkv"][:n].float()
    q, k, v = x.split([H * hd, kv * hd, kv * hd], dim=1)

    def queries(t):  # [n, H hd] -> [nb, kv, G C, hd]
        t = torch.nn.functional.pad(t, (0, 0, 0, nb * C - n)).view(nb, C, kv, G, hd)
        return t.permute(0, 2, 3, 1, 4).reshape(nb, kv, G * C, hd)

    def tokens(t):  # and back
        return t.view(nb, kv, G, C, hd).permute(0, 3, 1, 2, 4).reshape(nb * C, H * hd)[:n]

    def windows(t):  # [n, kv hd] -> [nb, kv, hd, C + W]: rows b C - W .. b C + C - 1
        t = torch.nn.functional.pad(t, (0, 0, W, nb * C - n))
        return t.view(-1, kv, hd).unfold(0, C + W, C).contiguous()

    i = torch.arange(nb * C, device=DEV).view(nb, C, 1)
    j = (torch.arange(nb, device=DEV) * C - W).view(nb, 1, 1) + torch.arange(C + W, device=DEV)
    first = torch.nn.functional.pad(start, (0, nb * C - n)).view(nb, C, 1)
    see = ((j <= i) & (j > i - W) & (j >= first) & (i < n))[:, None, None]
    at = first + torch.arange(max(1, S), device=DEV)  # the sinks of every query
    see_s = ((at <= i - W) & (i < n) & (S > 0))[:, None, None]
    at = at.clamp(max=n - 1)

    def score(a, kw, ks):  # a . key for both kinds of keys, [nb, kv, G, C, ...]
        near = torch.matmul(a, kw).view(nb, kv, G, C, C + W)
        far = torch.matmul(a.view(nb, kv, G, C, hd).permute(0, 3, 1, 2, 4), ks)
        return near, far.permute(0, 2, 3, 1, 4)

    def mix(near, far, kw, ks):  # sums of keys weighted by near and far, [nb, kv, G C, hd]
        t = torch.matmul(near.reshape(nb, kv, G * C, C + W), kw.transpose(2, 3).contiguous())
        u = torch.matmul(far.permute(0, 3, 1, 2, 4).contiguous(), ks.transpose(3, 4).contiguous())
        return t + u.permute(0, 2, 3, 1, 4).reshape(nb, kv, G * C, hd)

    def spread(near, far, a):  # the weights' sums over queries, [n, kv hd]
        t = torch.matmul(near.reshape(nb, kv, G * C, C + W).transpose(2, 3).contiguous(), a)
        acc = torch.zeros((W + nb * C, kv, hd), device=DEV)
        acc.index_add_(0, (j + W).reshape(-1), t.permute(0, 2, 1, 3).reshape(-1, kv, hd))
        acc = acc[W:W + n]
        u = torch.matmul(far.permute(0, 3, 1, 4, 2).contiguous(),
                         a.view(nb, kv, G, C, hd).permute(0, 3, 1, 2, 4).contiguous())
        acc.index_add_(0, at.reshape(-1), u.permute(0, 1, 3, 2, 4).reshape(-1, kv, hd))
        return acc.reshape(n, kv * hd)

    qb, kw, vw = queries(q), windows(k), windows(v)
    ks, vs = (t.reshape(n, kv, hd)[at].permute(0, 1, 3, 4, 2).contiguous() for t in (k, v))
    near, far = score(qb * scale, kw, ks)
    near, far = near.masked_fill(~see, -math.inf), far.masked_fill(~see_s, -math.inf)
    m = torch.maximum(near.amax(-1, keepdim=True), far.amax(-1, keepdim=True)).clamp(min=-1e30)
    near, far = torch.exp(near - m), torch.exp(far - m)
    total = (near.sum(-1, keepdim=True) + far.sum(-1, keepdim=True)).clamp(min=1e-30)
    near, far = near / total, far / total
    ob = mix(near, far, vw, vs)
    o, lse = torch.zeros_like(s["o"]), torch.zeros_like(s["lse"])
    o[:n] = tokens(ob).to(o.dtype)
    lse[:, :n] = (m + torch.log(total)).squeeze(-1).permute(1, 2, 0, 3).reshape(H, nb * C)[:, :n]
    if c["pass"] == "forward":
        return {"o": o, "lse": lse}
    db = queries(s["dout"][:n].float())
    D = (db * ob).sum(-1).view(nb, kv, G, C, 1)
    dv = spread(near, far, db)
    dp, dp_s = score(db, vw, vs)
    near, far = near * (dp - D) * scale, far * (dp_s - D) * scale
    dqkv = torch.zeros((rows, (H + 2 * kv) * hd), dtype=s["dqkv"].dtype, device=DEV)
    dqkv[:n] = torch.cat([tokens(mix(near, far, kw, ks)), spread(near, far, qb), dv], 1).to(dqkv.dtype)
    return {"o": o, "lse": lse, "dqkv": dqkv}


# ------------------------------------------------------------------ definitions, in 64 bits

def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "layernorm":
        x, g, b = s["x"].double(), s["g"].double(), s["b"].double()
        mu = x.sum(1) / c["d"]
        r = (((x - mu[:, None]) ** 2).sum(1) / c["d"] + EPS) ** -0.5
        xh = (x - mu[:, None]) * r[:, None]
        out = {"y": g * xh + b, "mean": mu, "rstd": r}
        if c["pass"] == "train":
            # through the row's sums: y depends on x by itself, by the mean and by the variance
            dy = s["dy"].double()
            t = g * dy
            dx = r[:, None] * t
            dx -= (r * t.sum(1) / c["d"])[:, None]
            dx -= xh * (r * torch.einsum("td,td->t", t, xh) / c["d"])[:, None]
            if s["dres"] is not None:
                dx += s["dres"].double()
            out |= {"dx": dx, "dg": torch.einsum("td,td->d", dy, xh), "db": dy.sum(0)}
        return out
    if c["op"] == "rope":
        half, T = c["hd"] // 2, c["tokens"]
        turn = torch.ones((T, half), dtype=torch.complex128, device=DEV)
        at = 0
        for a, n in enumerate(int(k) for k in c["sections"].split(",")):
            for i in range(n):
                f = math.exp(-math.log(c["base"]) * (i / n if c["freq"] == "axis" else at / half))
                p = s["pos"][a].double() * f
                turn[:, at] = torch.complex(torch.cos(p), torch.sin(p))
                at += 1
        if c["pass"] == "table":
            return {"cos": turn.real.contiguous(), "sin": turn.imag.contiguous()}
        x = s["x"].double().view(T, c["heads"], 2, half)
        z = torch.complex(x[:, :, 0], x[:, :, 1])
        z = z * (turn if c["pass"] == "forward" else turn.conj())[:, None]
        return {"y": torch.cat([z.real, z.imag], -1).view(T, -1)}
    return _attention_exact(s)


def _attention_exact(s):
    """Sequence by sequence and head by head, a few hundred queries at a time."""
    c = s["case"]
    H, kv, hd, W, S = c["heads"], c["kv"], c["hd"], c["window"], c["sinks"]
    G, train = H // kv, c["pass"] == "train"
    x, dout = s["qkv"].double(), s["dout"].double()
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    dx = torch.zeros_like(x)
    begin = 0
    for n in _lengths(c):
        row = slice(begin, begin + n)
        for h in range(H):
            cq, co = slice(h * hd, (h + 1) * hd), h // G
            ck = slice((H + co) * hd, (H + co + 1) * hd)
            cv = slice((H + kv + co) * hd, (H + kv + co + 1) * hd)
            q, k, v = x[row, cq], x[row, ck], x[row, cv]
            step = max(256, min(2048, W))
            for a in range(0, n, step):
                e = min(n, a + step)
                lo = max(0, a - W + 1)
                keys = torch.cat([torch.arange(0, min(S, lo), device=DEV), torch.arange(lo, e, device=DEV)])
                back = torch.arange(a, e, device=DEV)[:, None] - keys
                hide = (back < 0) | ((back >= W) & (keys >= S))
                z = (q[a:e] @ k[keys].T / math.sqrt(hd)).masked_fill(hide, -math.inf)
                L = torch.logsumexp(z, 1)
                p = torch.exp(z - L[:, None])
                y = p @ v[keys]
                o[begin + a:begin + e, cq], lse[h, begin + a:begin + e] = y, L
                if train:
                    do = dout[begin + a:begin + e, cq]
                    dz = p * (do @ v[keys].T - (do * y).sum(1, keepdim=True)) / math.sqrt(hd)
                    dx[begin + a:begin + e, cq] = dz @ k[keys]
                    dx[begin + keys, ck] += dz.T @ q[a:e]
                    dx[begin + keys, cv] += p.T @ do
        begin += n
    return {"o": o, "lse": lse, "dqkv": dx} if train else {"o": o, "lse": lse}
