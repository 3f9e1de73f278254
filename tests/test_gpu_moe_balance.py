"""The router's balance and z losses, per-expert counts and gradients against their formulas in 64
bits and against differences; and a mixture's whole pass in 8 bits.

Tolerances: a logit sums d products in fp32 (the pieces' products on the matrix cores, at most 9 for
each): D = (d/32 * 9 + 16) * 2^-24 * sum |n wr| at most; probs are off by exp(2 D) - 1 relative and 2^-20
for exp and the sum; lse by D + 2^-22 (1 + |lse|). dl is formed from fp32 numbers: its terms (each
bounded by its own magnitude) times the relative error of p, f and lse, 2^-18 + 4 D in all. dn and dWr
sum E and N such terms, with 2^-24 per addition, and dn's own rounding.
"""
import pytest
import torch

from paper_2606_11169_amd import libchunk as lc

pytestmark = pytest.mark.gpu

DT = {"fp32": (lc.LC_FP32, torch.float32), "bf16": (lc.LC_BF16, torch.bfloat16), "fp16": (lc.LC_FP16, torch.float16)}
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
COEF, Z = 0.02, 0.003


def inputs(T, d, E, n, w, seed, masked=False, std=0.05):
    g = torch.Generator().manual_seed(seed)
    s = {"n": torch.randn(T, d, generator=g).to(DT[n][1]), "wr": (torch.randn(E, d, generator=g) * std).to(DT[w][1])}
    l = s["n"].double() @ s["wr"].double().T
    top = torch.topk(l, 2, dim=1)
    s["sel"], s["w"] = top.indices.int(), torch.softmax(top.values, 1).float()
    s["dw"] = torch.randn(T, 2, generator=g) * 0.1
    s["mask"] = (torch.rand(T, generator=g) < 0.7).to(torch.uint8) if masked else None
    s["dres"] = torch.randn(T, d, generator=g) * 0.01
    return s


def reference(s, E, pair=True, dres=True):
    n, wr = s["n"].double(), s["wr"].double()
    T = n.shape[0]
    live = s["mask"].bool() if s["mask"] is not None else torch.ones(T, dtype=torch.bool)
    N = int(live.sum())
    n = torch.where(live[:, None], n, 0.0)
    l = n @ wr.T
    mag = n.abs() @ wr.abs().T
    p = torch.softmax(l, 1) * live[:, None]
    lse = torch.logsumexp(l, 1) * live
    sel = s["sel"].long()
    ok = (sel >= 0) & (sel < E) & live[:, None]
    ok[:, 1] &= sel[:, 1] != sel[:, 0]
    one = torch.nn.functional.one_hot(sel.clamp(0, E - 1), E) * ok[:, :, None]
    counts = one.sum((0, 1))
    f = counts.double() / max(1, 2 * N)
    r = {"p": p, "lse": lse, "counts": torch.cat([counts, torch.tensor([N])]).int(), "mag": mag}
    r["loss"] = torch.tensor([E * (f * p.sum(0)).sum() / max(1, N), (lse ** 2).sum() / max(1, N)])
    rn = 1.0 / N if N else 0.0
    terms = [COEF * E * rn * p * f, COEF * E * rn * p * (p * f).sum(1, keepdim=True), 2 * Z * rn * lse[:, None] * p]
    dl = terms[0] - terms[1] + terms[2]
    size = terms[0] + terms[1] + terms[2].abs()
    if pair:
        w, dw = (torch.where(ok, s[k].double(), 0.0) for k in ("w", "dw"))
        gate = w * (dw - (w * dw).sum(1, keepdim=True))
        dl = dl + (one * gate[:, :, None]).sum(1)
        size = size + (one * (w * (dw.abs() + (w * dw.abs()).sum(1, keepdim=True)))[:, :, None]).sum(1)
    r["dl"], r["size"] = dl, size
    r["dn"] = dl @ wr + (s["dres"].double() if dres else 0)
    r["dwr"] = dl.T @ n
    r["dn_size"], r["dwr_size"] = size @ wr.abs(), size.T @ n.abs()
    return r


def call(s, E, n, w, dn="fp32", dres=None, pair=True, store=1, dwr0=None, scratch=None, stream=None):
    T, d = s["n"].shape
    g = {k: (v.cuda() if v is not None else None) for k, v in s.items()}
    o = {"p": torch.full((T, E), 9.0, device="cuda"), "lse": torch.full((T,), 9.0, device="cuda"),
         "counts": torch.full((E + 1,), 9, dtype=torch.int32, device="cuda"), "loss": torch.full((2,), 9.0, device="cuda"),
         "dn": torch.full((T, d), 9.0, dtype=DT[dn][1], device="cuda"),
         "dwr": dwr0.cuda() if dwr0 is not None else torch.full((E, d), 9.0, device="cuda")}
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    scratch = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") if scratch is None else scratch
    lc.lc_moe_balance_forward(T, d, E, g["n"], g["wr"], g["sel"], o["p"], o["lse"], o["counts"], o["loss"], scratch,
                              size, DT[n][0], DT[w][0], mask=g["mask"], stream=stream)
    lc.lc_moe_balance_backward(T, d, E, g["n"], g["wr"], g["sel"], o["p"], o["lse"], o["counts"], COEF, Z, o["dn"],
                               o["dwr"], scratch, size, DT[n][0], DT[w][0], DT[dn][0],
                               dres=g["dres"].to(DT[dres][1]) if dres else None, dres_dtype=DT[dres or "fp32"][0],
                               w=g["w"] if pair else None, dw=g["dw"] if pair else None, mask=g["mask"], store_dwr=store,
                               stream=stream)
    return o


def check(o, r, d, dn="fp32", add=None):
    o = {k: v.cpu().double() if v.is_floating_point() else v.cpu() for k, v in o.items()}
    D = (d / 32 * 9 + 16) * 2.0 ** -24 * r["mag"].amax(1, keepdim=True)
    assert torch.equal(o["counts"], r["counts"])
    rel = torch.expm1(2 * D) + 2.0 ** -20
    # (fp32 has no normal numbers below 2^-126: what exp gives there may be a subnormal's step off, or 0)
    assert bool(((o["p"] - r["p"]).abs() <= rel * r["p"] + 2.0 ** -126).all())
    assert bool(((o["lse"] - r["lse"]).abs() <= D[:, 0] + 2.0 ** -22 * (1 + r["lse"].abs())).all())
    worst = rel.max() if len(rel) else 0.0
    assert bool(((o["loss"] - r["loss"]).abs() <= 4 * (worst + 2.0 ** -20) * (r["loss"].abs() + 1e-30)).all())
    T, E = r["p"].shape
    off = rel * 4 + 2.0 ** -18
    tol = off * r["dn_size"] + (E + 8) * 2.0 ** -24 * r["dn_size"] + (HALF_STEP[dn] + 2.0 ** -24) * r["dn"].abs() + 1e-30
    assert bool(((o["dn"] - r["dn"]).abs() <= tol).all()), ((o["dn"] - r["dn"]).abs() / tol).max()
    want = r["dwr"] + (add.double() if add is not None else 0)
    tol = ((worst * 4 + 2.0 ** -18) + (T + 8) * 2.0 ** -24) * r["dwr_size"] + 2.0 ** -23 * want.abs() + 1e-30
    assert bool(((o["dwr"] - want).abs() <= tol).all()), ((o["dwr"] - want).abs() / tol).max()


@pytest.mark.parametrize("n,w", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32"), ("fp32", "bf16"),
                                 ("fp16", "fp32"), ("bf16", "fp16"), ("fp32", "fp16"), ("fp16", "bf16")])
@pytest.mark.parametrize("E", [2, 8, 17, 33, 64])
def test_types_and_experts(E, n, w):
    T, d = 150, 200
    s = inputs(T, d, E, n, w, E, masked=E != 8)
    check(call(s, E, n, w, dres="fp32"), reference(s, E), d)


@pytest.mark.parametrize("T,d,E,masked", [(1, 8, 2, False), (1, 4096, 64, False), (31, 72, 5, True), (32, 128, 8, False),
                                          (33, 136, 8, True), (700, 1032, 8, False), (3000, 256, 40, True),
                                          (9001, 64, 3, False), (8200, 512, 64, True)])
def test_shapes(T, d, E, masked):
    s = inputs(T, d, E, "bf16", "bf16", T + E, masked)
    check(call(s, E, "bf16", "bf16", dn="bf16", dres="bf16"), {**reference({**s, "dres": s["dres"].bfloat16()}, E)}, d, "bf16")


def test_accumulate_and_parts():
    """dWr added to what is there; no pair gradient, no residual; dn or dWr alone gives the same bits."""
    T, d, E = 300, 264, 8
    s = inputs(T, d, E, "bf16", "fp32", 4)
    start = torch.randn(E, d, generator=torch.Generator().manual_seed(1))
    o = call(s, E, "bf16", "fp32", store=0, dwr0=start)
    check(o, reference(s, E, dres=False), d, add=start)
    check(call(s, E, "bf16", "fp32", pair=False), reference(s, E, pair=False, dres=False), d)
    g = {k: v.cuda() for k, v in s.items() if v is not None}
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    dn, dwr = torch.empty(T, d, device="cuda"), start.cuda()
    common = dict(w=g["w"], dw=g["dw"])
    args = (T, d, E, g["n"], g["wr"], g["sel"], o["p"], o["lse"], o["counts"], COEF, Z)
    lc.lc_moe_balance_backward(*args, dn, None, None, 0, lc.LC_BF16, lc.LC_FP32, lc.LC_FP32, **common)
    lc.lc_moe_balance_backward(*args, None, dwr, scratch, size, lc.LC_BF16, lc.LC_FP32, lc.LC_FP32, **common)
    assert torch.equal(dn, o["dn"]) and torch.equal(dwr, o["dwr"])


def test_selection_edges():
    """Pairs out of range or twice the same expert are not counted and carry no gradient."""
    T, d, E = 70, 64, 8
    s = inputs(T, d, E, "bf16", "bf16", 6)
    s["sel"][3] = torch.tensor([5, 5])
    s["sel"][4] = torch.tensor([-1, 2])
    s["sel"][5] = torch.tensor([3, 8])
    s["sel"][6] = torch.tensor([-7, 2 ** 31 - 1])
    check(call(s, E, "bf16", "bf16"), reference(s, E, dres=False), d)


def test_masked_tokens_reach_nothing():
    """Infinities and NaN in tokens that do not count; all tokens masked; none."""
    T, d, E = 100, 136, 8
    s = inputs(T, d, E, "bf16", "fp32", 7, masked=True)
    o = call(s, E, "bf16", "fp32", dres="fp32")
    off = ~s["mask"].bool()
    s["n"][off] = float("nan")
    s["dw"][off] = float("inf")
    s["n"][off.nonzero()[0, 0], 5] = float("inf")
    s["w"][off] = float("nan")
    s["sel"][off] = 1 << 30
    o2 = call(s, E, "bf16", "fp32", dres="fp32")
    for k in o:
        assert torch.equal(o[k], o2[k]), k
    assert bool((o["p"].cpu()[off] == 0).all()) and torch.equal(o["dn"].cpu()[off], s["dres"][off])
    s["mask"] = torch.zeros(T, dtype=torch.uint8)
    o = call(s, E, "bf16", "fp32", dres="fp32")
    assert int(o["counts"].abs().sum()) == 0 and float(o["loss"].abs().sum()) == 0 and float(o["dwr"].abs().sum()) == 0
    assert torch.equal(o["dn"].cpu(), s["dres"]) and float(o["p"].abs().sum()) == 0


def test_no_tokens():
    E, d = 8, 64
    counts, loss = torch.full((E + 1,), 5, dtype=torch.int32, device="cuda"), torch.full((2,), 5.0, device="cuda")
    dwr = torch.full((E, d), 5.0, device="cuda")
    size = lc.lc_moe_balance_scratch_bytes(0, d, E)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    lc.lc_moe_balance_forward(0, d, E, None, None, None, None, None, counts, loss, scratch, size, lc.LC_BF16, lc.LC_BF16)
    assert int(counts.abs().sum()) == 0 and float(loss.abs().sum()) == 0
    for store, want in ((0, 5.0), (1, 0.0)):
        lc.lc_moe_balance_backward(0, d, E, None, None, None, None, None, counts, COEF, Z, None, dwr, scratch, size,
                                   lc.LC_BF16, lc.LC_BF16, lc.LC_FP32, store_dwr=store)
        assert bool((dwr == want).all())


def test_nan_token():
    """A NaN in a token that counts reaches its own rows of probs and dn, and the sums, not other rows."""
    T, d, E = 64, 64, 8
    s = inputs(T, d, E, "bf16", "bf16", 8)
    a = call(s, E, "bf16", "bf16")
    s["n"][10, 3] = float("nan")
    b = call(s, E, "bf16", "bf16")
    keep = torch.arange(T) != 10
    assert torch.equal(a["p"].cpu()[keep], b["p"].cpu()[keep]) and bool(torch.isnan(b["p"][10]).all())
    assert bool(torch.isnan(b["loss"]).all()) and torch.equal(a["counts"], b["counts"])
    assert bool(torch.isnan(b["dn"][10]).all()) and torch.equal(a["dn"].cpu()[keep], b["dn"].cpu()[keep])
    assert bool(torch.isnan(b["dwr"]).any(1).all())


def test_large_logits():
    """Logits of hundreds: no overflow in exp."""
    T, d, E = 40, 64, 8
    s = inputs(T, d, E, "fp32", "fp32", 9, std=20.0)
    check(call(s, E, "fp32", "fp32"), reference(s, E, dres=False), d)


def test_gradient_against_differences():
    """d loss / d n and d Wr against central differences of the forward's formula in 64 bits."""
    T, d, E = 9, 16, 4
    s = inputs(T, d, E, "fp32", "fp32", 10, std=0.5)
    o = call(s, E, "fp32", "fp32", pair=False)

    def loss(n, wr):
        r = reference({**s, "n": n, "wr": wr}, E, pair=False, dres=False)["loss"]
        return float(COEF * r[0] + Z * r[1])

    n, wr, h = s["n"].double(), s["wr"].double(), 1e-5
    for (x, got) in ((n, o["dn"]), (wr, o["dwr"])):
        got = got.double().cpu()
        for i in range(x.shape[0]):
            for j in range(0, x.shape[1], 3):
                keep = float(x[i, j])
                x[i, j] = keep + h
                plus = loss(n, wr)
                x[i, j] = keep - h
                minus = loss(n, wr)
                x[i, j] = keep
                # differences: h^2 of third derivatives (below 1) and rounding of the losses over h
                assert abs((plus - minus) / (2 * h) - float(got[i, j])) <= 1e-9 + 2.0 ** -16 * float(got.abs().max())


# ------------------------------------------------------------------ graphs and streams

def test_captured_graphs_share_a_workspace():
    """Two graphs of different sizes on one scratch and one capture stream, replayed in turn with
    eager work between, give the eager results each time."""
    E = 8
    cases = [inputs(600, 264, E, "bf16", "bf16", 1), inputs(90, 512, E, "bf16", "bf16", 2, True)]
    size = max(lc.lc_moe_balance_scratch_bytes(*c["n"].shape, E) for c in cases)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    st, graphs = torch.cuda.Stream(), []
    eager = [call(c, E, "bf16", "bf16", dres="fp32") for c in cases]
    for c in cases:
        T, d = c["n"].shape
        g = {k: (v.cuda() if v is not None else None) for k, v in c.items()}
        o = {"p": torch.zeros(T, E, device="cuda"), "lse": torch.zeros(T, device="cuda"),
             "counts": torch.zeros(E + 1, dtype=torch.int32, device="cuda"), "loss": torch.zeros(2, device="cuda"),
             "dn": torch.zeros(T, d, device="cuda"), "dwr": torch.zeros(E, d, device="cuda")}
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            cur = torch.cuda.current_stream()
            lc.lc_moe_balance_forward(T, d, E, g["n"], g["wr"], g["sel"], o["p"], o["lse"], o["counts"], o["loss"],
                                      scratch, size, lc.LC_BF16, lc.LC_BF16, mask=g["mask"], stream=cur)
            lc.lc_moe_balance_backward(T, d, E, g["n"], g["wr"], g["sel"], o["p"], o["lse"], o["counts"], COEF, Z, o["dn"],
                                       o["dwr"], scratch, size, lc.LC_BF16, lc.LC_BF16, lc.LC_FP32, dres=g["dres"],
                                       dres_dtype=lc.LC_FP32, w=g["w"], dw=g["dw"], mask=g["mask"], store_dwr=1, stream=cur)
        graphs.append((graph, o, g))
    for _ in range(4):
        for (graph, o, _), want in zip(graphs, eager):
            for t in o.values():
                t.zero_()
            scratch.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            for k in o:
                assert torch.equal(o[k], want[k]), k
            (scratch[:1000].float() + 1).sum().item()


def test_streams():
    """Calls on three streams at once, each with its own scratch."""
    E, cases = 8, [inputs(500 + 64 * i, 136, 8, "bf16", "bf16", i) for i in range(3)]
    eager = [call(c, E, "bf16", "bf16") for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for c, st in zip(cases, streams):
        with torch.cuda.stream(st):
            got.append(call(c, E, "bf16", "bf16", stream=st))
    torch.cuda.synchronize()
    for a, b in zip(eager, got):
        for k in a:
            assert torch.equal(a[k], b[k]), k


# ------------------------------------------------------------------ a mixture's pass in 8 bits

def test_far_tokens():
    """Tokens whose offsets pass 2^31 values: zeros but for a few, which decide what is checked."""
    T, d, E, few = 40000, 1 << 16, 4, [0, 7, 32767, 32768, 32769, 39990, 39999]
    s = inputs(len(few), d, E, "bf16", "bf16", 3, std=0.005)
    n = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    n[torch.tensor(few, device="cuda")] = s["n"].cuda()
    z = lambda *k, t=torch.float32: torch.zeros(*k, dtype=t, device="cuda")  # noqa: E731
    sel = torch.arange(2 * T, dtype=torch.int32).remainder(E).view(T, 2).cuda()
    mask = z(T, t=torch.uint8)
    mask[torch.tensor(few, device="cuda")] = 1
    wr = s["wr"].cuda()
    p, lse, counts, loss = z(T, E), z(T), z(E + 1, t=torch.int32), z(2)
    dn, dwr = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), z(E, d)
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    scratch = z(size, t=torch.uint8)
    BF = lc.LC_BF16
    lc.lc_moe_balance_forward(T, d, E, n, wr, sel, p, lse, counts, loss, scratch, size, BF, BF, mask=mask)
    lc.lc_moe_balance_backward(T, d, E, n, wr, sel, p, lse, counts, COEF, Z, dn, dwr, scratch, size, BF, BF, BF,
                               mask=mask, store_dwr=1)
    at = torch.tensor(few, device="cuda")
    t = {"n": s["n"], "wr": s["wr"], "sel": sel[at].cpu(), "w": s["w"], "dw": s["dw"], "mask": None,
         "dres": torch.zeros(len(few), d)}
    check({"p": p[at], "lse": lse[at], "counts": counts, "loss": loss, "dn": dn[at], "dwr": dwr},
          reference(t, E, pair=False, dres=False), d, "bf16")
    dn[at] = 0
    assert not bool(dn.any()) and float(p.sum()) == pytest.approx(len(few), rel=1e-5)


def up(n, to):
    return -(-n // to) * to


def quantized(T, d, x, xd, q, layouts="rc", block=1, offsets=None, n_groups=0, **k):
    """Bytes and scales of lc_fp8_quantize, and what they stand for in 64 bits (rows [T, d], columns
    [d, columns])."""
    cols = lc.lc_fp8_padded_rows(T, n_groups)
    mk = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    o = {"q": mk(T, up(d, 16)), "s": mk(up(d, 128) // 128, up(-(-T // block), 4)), "qt": mk(d, cols),
         "st": mk(cols // 128, up(-(-d // block), 4))}
    lc.lc_fp8_quantize(T, d, x, xd, q, q=o["q"], ld_q=o["q"].stride(0), scale=o["s"], ld_scale=o["s"].stride(0), qt=o["qt"],
                       ld_qt=cols, scale_t=o["st"], ld_scale_t=o["st"].stride(0), block_rows=block, group_offsets=offsets,
                       n_groups=n_groups, **k)
    t = torch.float8_e4m3fn if q == lc.LC_FP8_E4M3 else torch.float8_e5m2

    def stand(b, s, r, c):
        f = torch.exp2(s.cpu().double() - 127).T.repeat_interleave(block, 0)[:r].repeat_interleave(128, 1)[:, :c]
        return b.cpu().view(t).float().double()[:, :c] * f

    return o, stand(o["q"], o["s"], T, d), stand(o["qt"], o["st"], d, cols)


def close(got, want, mag, half, K):
    """A product's result of 16 bits or 32: see test_gpu_fp8."""
    got = got.double().cpu()
    tol = (8 * 2.0 ** -13 if half > 2.0 ** -20 else K / 32 * 6 * 2.0 ** -24) * mag + half * want.abs() + 2.0 ** -20 * mag
    assert bool(((got - want).abs() <= tol).all()), ((got - want).abs() / tol).max()


def test_mixture_pass():
    """Router, balance loss, dispatch, the experts' rows gathered and quantised, both expert products,
    and back: input gradients and weight gradients, every product against 64 bits on the operands
    it was given, and the quantised operands against the values they were made of."""
    T, d, E, f = 333, 256, 8, 192
    g = torch.Generator().manual_seed(21)
    n = torch.randn(T, d, generator=g).bfloat16().cuda()
    wr = (torch.randn(E, d, generator=g) * 0.05).bfloat16().cuda()
    W1 = (torch.randn(E, f, d, generator=g) * 0.05).bfloat16().cuda()
    W2 = (torch.randn(E, d, f, generator=g) * 0.05).bfloat16().cuda()
    BF, E4, E5 = lc.LC_BF16, lc.LC_FP8_E4M3, lc.LC_FP8_E5M2
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    sel, w = i32(T, 2), torch.zeros(T, 2, device="cuda")
    lc.lc_moe_route(T, d, E, n, wr, sel, w, BF, BF)
    off, perm, wrow, rowpos = i32(E + 1), i32(2 * T), torch.zeros(2 * T, device="cuda"), i32(T, 2)
    lc.lc_moe_dispatch(T, E, sel, w, off, perm, wrow, rowpos)
    p, lse, counts, loss = torch.zeros(T, E, device="cuda"), torch.zeros(T, device="cuda"), i32(E + 1), torch.zeros(2, device="cuda")
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    lc.lc_moe_balance_forward(T, d, E, n, wr, sel, p, lse, counts, loss, scratch, size, BF, BF)
    assert torch.equal(counts[:E], off[1:] - off[:-1]) and int(counts[E]) == T

    R, o = 2 * T, off.cpu().tolist()
    xq, xv, xtv = quantized(R, d, n, BF, E4, row_index=perm, x_rows=T, offsets=off, n_groups=E)
    rows = n.cpu().double()[perm.cpu().long()]
    assert bool(((xv - rows).abs() <= 2.0 ** -4 * rows.abs() + 2.0 ** -10 * rows.abs().amax(1, keepdim=True) / 224).all())
    w1 = [quantized(f, d, W1[e].contiguous(), BF, E4, block=128) for e in range(E)]
    w2 = [quantized(d, f, W2[e].contiguous(), BF, E4, block=128) for e in range(E)]

    def grouped(a, ws, N, K, key, skey, a_dtype=E4):
        C = torch.zeros(R, N, dtype=torch.bfloat16, device="cuda")
        B, S = torch.cat([x[0][key] for x in ws]), torch.cat([x[0][skey] for x in ws])
        lc.lc_gemm_fp8(lc.LC_EPI_STORE, R, N, K, a["q"], a["q"].stride(0), a["s"], a["s"].stride(0), B, B.stride(0), S,
                       S.stride(0), C, N, a_dtype=a_dtype, group_mode=lc.LC_GROUP_ROWS, n_groups=E, group_offsets=off,
                       group_stride_b=N * B.stride(0), group_stride_b_scale=ws[0][0][skey].numel())
        return C

    def per_expert(C, av, wv):
        for e in range(E):
            x = av[o[e]:o[e + 1]]
            close(C[o[e]:o[e + 1]], x @ wv[e].T, x.abs() @ wv[e].abs().T, 2.0 ** -8, x.shape[1])

    h = grouped(xq, w1, f, d, "q", "s")
    per_expert(h, xv, [x[1] for x in w1])
    act = torch.nn.functional.silu(h.float()).bfloat16()
    aq, av, atv = quantized(R, f, act, BF, E4, offsets=off, n_groups=E)
    y = grouped(aq, w2, d, f, "q", "s")
    per_expert(y, av, [x[1] for x in w2])

    # back: the gradient at the experts' outputs is the tokens', gathered and weighted
    dy = (torch.randn(T, d, generator=g) * 1e-3).bfloat16().cuda()
    gq, gv, gtv = quantized(R, d, dy, BF, E5, row_index=perm, x_rows=T, row_weight=wrow, offsets=off, n_groups=E)
    da = grouped(gq, w2, f, d, "qt", "st", a_dtype=E5)  # W2's columns: [f, d], blocks of 128 x 128
    per_expert(da, gv, [x[2][:, :d] for x in w2])
    # dW2[e] = sum over its rows of dy^T act
    K = lc.lc_fp8_padded_rows(R, E)
    for c, code, half in ((torch.bfloat16, BF, 2.0 ** -8), (torch.float32, lc.LC_FP32, 2.0 ** -24)):
        dW = torch.zeros(E, d, f, dtype=c, device="cuda")
        lc.lc_gemm_fp8(lc.LC_EPI_STORE, d, f, K, gq["qt"], K, gq["st"], gq["st"].stride(0), aq["qt"], K, aq["st"],
                       aq["st"].stride(0), dW, f, a_dtype=E5, c_dtype=code, b_block_rows=1, group_mode=lc.LC_GROUP_K,
                       n_groups=E, group_offsets=off, group_stride_c=d * f)
        at = 0
        for e in range(E):
            m = o[e + 1] - o[e]
            a, b = gtv[:, at:at + m], atv[:, at:at + m]
            close(dW[e], a @ b.T, a.abs() @ b.abs().T, half, m)
            at += up(m, 128)
    # the router's gradient: balance, z loss and the gates'
    eo = y.float()
    dw = torch.stack([(dy.float() * eo[rowpos[:, k].long()]).sum(1) for k in (0, 1)], 1).contiguous()
    dn, dwr = torch.zeros(T, d, device="cuda"), torch.zeros(E, d, device="cuda")
    lc.lc_moe_balance_backward(T, d, E, n, wr, sel, p, lse, counts, COEF, Z, dn, dwr, scratch, size, BF, BF, lc.LC_FP32,
                               w=w, dw=dw, store_dwr=1)
    s = {"n": n.cpu(), "wr": wr.cpu(), "sel": sel.cpu(), "w": w.cpu(), "dw": dw.cpu(), "mask": None, "dres": torch.zeros(T, d)}
    check({"p": p, "lse": lse, "counts": counts, "loss": loss, "dn": dn, "dwr": dwr}, reference(s, E), d)


# ------------------------------------------------------------------ values of more bits than bf16's

def single(n, wr, T, d, E, n_dt, w_dt, x):
    """dn and dwr of one dl: token 0 of its own, with N = 1, lse = x and probs 1 at expert 0, of z_coef 0.5
    and coef 0: dl[0, 0] is x exactly, all others 0."""
    p, lse = torch.zeros(T, E, device="cuda"), torch.zeros(T, device="cuda")
    p[0, 0], lse[0] = 1.0, float(x)
    counts = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    counts[E] = 1
    dn, dwr = torch.empty(T, d, device="cuda"), torch.empty(E, d, device="cuda")
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    sel = torch.tensor([0, 1], dtype=torch.int32).repeat(T, 1).cuda()
    lc.lc_moe_balance_backward(T, d, E, n.cuda(), wr.cuda(), sel, p, lse, counts, 0.0, 0.5, dn, dwr,
                               torch.empty(size, dtype=torch.uint8, device="cuda"), size, DT[n_dt][0], DT[w_dt][0], lc.LC_FP32,
                               store_dwr=1)
    return dn.cpu().double(), dwr.cpu().double()


@pytest.mark.parametrize("n,w", [("fp32", "fp32"), ("fp32", "fp16"), ("fp16", "fp32"), ("fp16", "fp16"), ("fp32", "bf16"),
                                 ("bf16", "fp32"), ("bf16", "bf16")])
def test_products_keep_fp32(n, w):
    """Single products (one value of n meets one of wr, or one dl): fp32's pieces, rounded to nearest,
    leave out two products of 2^-8 by 2^-17 of the values' powers of two (by fp16's two pieces one of
    2^-7 by 2^-17): 2^-24 of the product at most; then the
    smaller pieces' sum is rounded at 2^-7 of the product or below, and the last addition to fp32's step
    (2^-23, if it is not to nearest). So (1 + 2 + 2^-5) 2^-24; where pieces are cut, up to 7.9 are left out."""
    T, d, E = 64, 64, 2
    tol = (1 + 2 + 2.0 ** -5) * 2.0 ** -24
    g = torch.Generator().manual_seed(3)
    mk = lambda *s: 1 + torch.rand(*s, generator=g) * 0.999  # noqa: E731
    value = {"fp32": 1.0078124, "fp16": 1.0068359375, "bf16": 1.0078125}  # (many low bits)
    for turn in range(4):
        nv = torch.full((d,), value[n]) if turn == 0 else mk(d)
        wv = torch.full((d,), value[w]) if turn == 0 else mk(d)
        nv, wv = nv.to(DT[n][1]), wv.to(DT[w][1])
        # forward: token t has value t alone; expert 1's weights are 0. Logits of some hundreds, so that
        # lse is the logit itself
        N, W = torch.zeros(T, d, dtype=nv.dtype), torch.zeros(E, d, dtype=wv.dtype)
        N[torch.arange(T), torch.arange(T)] = nv * 16
        W[0] = wv * 16
        s = {"n": N, "wr": W, "sel": torch.tensor([[0, 1]] * T, dtype=torch.int32), "mask": None, "w": None, "dw": None,
             "dres": None}
        o = call(s, E, n, w, pair=False)
        want = nv.double() * wv.double() * 256
        assert float(((o["lse"].cpu().double() - want).abs() / (tol * want)).max()) <= 1.0
        # backward: dl = x, times wr and n
        x = (1.0078124 if turn == 0 else mk(1)) * torch.ones(1)
        N = torch.zeros(T, d, dtype=nv.dtype)
        N[0] = nv
        dn, dwr = single(N, W, T, d, E, n, w, x)
        for got, other in ((dn[0], W[0].double()), (dwr[0], nv.double())):
            want = float(x) * other
            assert float(((got - want).abs() / (tol * want)).max()) <= 1.0
        assert float(dn[1:].abs().max()) == 0 and float(dwr[1].abs().max()) == 0


def test_largest_values():
    """Values next to fp32's largest, whose nearest bf16 is infinite, times small ones."""
    T, d, E = 3, 8, 2
    top = torch.tensor([0x7F7FFFFF, 0x7F7F8000, 0x7F7F7FFF, 0x7F000001], dtype=torch.int32).view(torch.float32)
    n, wr = torch.zeros(T, d), torch.zeros(E, d)
    n[0, :4], n[1, :4] = top, -top
    wr[0, :4] = top
    dn, dwr = single(n, wr, T, d, E, "fp32", "fp32", 2.0 ** -20)
    want = torch.zeros(E, d, dtype=torch.float64)
    want[0, :4] = top.double() * 2.0 ** -20
    assert torch.equal(dwr, want) and torch.equal(dn[0], want[0])
    wr[0, :4] = torch.tensor([2.0 ** -120, 0, 0, 0])
    s = {"n": n, "wr": wr, "sel": torch.tensor([[0, 1]] * T, dtype=torch.int32), "mask": None, "w": None, "dw": None,
         "dres": None}
    o = call(s, E, "fp32", "fp32", pair=False)
    assert float(o["lse"][0]) == float(top[0].double() * 2.0 ** -120)


def quiet(bits):
    """An fp32 value of these bits."""
    return torch.tensor([bits], dtype=torch.int32).view(torch.float32)


@pytest.mark.parametrize("bits", [0x7F800001, 0x7F80FFFF, -0x7FFFFF, 0x7FC00000], ids=hex)
def test_nan_of_any_payload(bits):
    """A NaN of fp32 whose bits all lie below bf16's is a NaN in every result that it reaches."""
    T, d, E = 70, 64, 8
    s = inputs(T, d, E, "fp32", "fp32", 8)
    a = call(s, E, "fp32", "fp32")
    keep = torch.arange(T) != 10
    # (values through integers: moving a signalling NaN as a float may quiet it)
    s["n"].view(torch.int32)[10, 3] = bits
    s["wr"][:, 3] = -s["wr"][:, 3].abs()  # as an infinity it would leave probabilities of 0
    a = call({**s, "n": torch.where(torch.isnan(s["n"]), 0.0, s["n"])}, E, "fp32", "fp32")
    b = call(s, E, "fp32", "fp32")
    assert torch.equal(a["p"].cpu()[keep], b["p"].cpu()[keep]) and bool(torch.isnan(b["p"][10]).all())
    assert bool(torch.isnan(b["loss"]).all()) and bool(torch.isnan(b["dn"][10]).all())
    # given finite probs, n's NaN reaches dwr's column alone
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    scratch, dwr = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(E, d, device="cuda")
    args = (T, d, E, s["n"].cuda(), s["wr"].cuda(), s["sel"].cuda(), a["p"], a["lse"], a["counts"], COEF, Z)
    lc.lc_moe_balance_backward(*args, None, dwr, scratch, size, lc.LC_FP32, lc.LC_FP32, lc.LC_FP32, store_dwr=1)
    assert bool(torch.isnan(dwr[:, 3]).all()) and not bool(torch.isnan(dwr[:, torch.arange(d) != 3]).any())
    # a weight: expert 2's logits are NaN, not -inf
    s = inputs(T, d, E, "fp32", "fp32", 8)
    s["n"][:, 5] = s["n"][:, 5].abs() * (1 if bits < 0 else -1) - (0 if bits < 0 else 1e-3)
    s["wr"].view(torch.int32)[2, 5] = bits
    b = call(s, E, "fp32", "fp32")
    assert bool(torch.isnan(b["p"]).all()) and bool(torch.isnan(b["lse"]).all())
    dn = b["dn"]
    lc.lc_moe_balance_backward(T, d, E, s["n"].cuda(), s["wr"].cuda(), s["sel"].cuda(), a["p"], a["lse"], a["counts"], COEF, Z,
                               dn, None, None, 0, lc.LC_FP32, lc.LC_FP32, lc.LC_FP32)
    assert bool(torch.isnan(dn[:, 5]).all()) and not bool(torch.isnan(dn[:, torch.arange(d) != 5]).any())


@pytest.mark.parametrize("n,w", [("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32"), ("fp32", "bf16"),
                                 ("fp16", "fp32"), ("bf16", "fp16"), ("fp32", "fp16"), ("fp16", "bf16")])
@pytest.mark.parametrize("E", [3, 40])
def test_infinite_weights(E, n, w):
    """An expert whose logits are -inf has probability 0, and the others what they have without it, in
    every type; an infinite value of a token leaves its row NaN (inf - inf)."""
    T, d = 90, 200
    s = inputs(T, d, E, n, w, E)
    s["n"][:, 7] = s["n"][:, 7].abs() + 0.125
    s["n"][4, 7] = 1.0  # (a value of one bf16 piece)
    s["wr"][1, 7] = -float("inf")
    o = call(s, E, n, w)
    keep = [e for e in range(E) if e != 1]
    l = s["n"].double() @ s["wr"][keep].double().T
    p, lse = torch.softmax(l, 1), torch.logsumexp(l, 1)
    D = (d / 32 * 9 + 16) * 2.0 ** -24 * (s["n"].double().abs() @ s["wr"][keep].double().abs().T).amax(1, keepdim=True)
    rel = torch.expm1(2 * D) + 2.0 ** -20
    got = o["p"].cpu().double()
    assert bool((got[:, 1] == 0).all()) and bool(((got[:, keep] - p).abs() <= rel * p + 2.0 ** -126).all())
    assert bool(((o["lse"].cpu().double() - lse).abs() <= D[:, 0] + 2.0 ** -22 * (1 + lse.abs())).all())
    s = inputs(T, d, E, n, w, E)
    s["n"][4, 7] = float("inf")
    o = call(s, E, n, w)
    assert bool(torch.isnan(o["p"][4]).all()) and bool(torch.isfinite(o["p"][torch.arange(T) != 4]).all())


def test_infinite_weights_in_the_backward():
    """What an infinite weight reaches is not finite, and nothing else changes."""
    T, d, E = 70, 64, 8
    for n, w in (("bf16", "bf16"), ("fp32", "fp32"), ("fp16", "fp16"), ("bf16", "fp32")):
        s = inputs(T, d, E, n, w, 8)
        a = call(s, E, n, w)
        s["wr"][2, 5] = float("inf")
        size = lc.lc_moe_balance_scratch_bytes(T, d, E)
        dn, dwr = torch.empty(T, d, device="cuda"), torch.empty(E, d, device="cuda")
        lc.lc_moe_balance_backward(T, d, E, s["n"].cuda(), s["wr"].cuda(), s["sel"].cuda(), a["p"], a["lse"], a["counts"], COEF, Z,
                                   dn, dwr, torch.empty(size, dtype=torch.uint8, device="cuda"), size, DT[n][0], DT[w][0],
                                   lc.LC_FP32, w=s["w"].cuda(), dw=s["dw"].cuda(), store_dwr=1)
        keep = torch.arange(d) != 5
        assert not bool(torch.isfinite(dn[:, 5]).any())
        assert torch.equal(dn[:, keep], a["dn"][:, keep]) and torch.equal(dwr, a["dwr"])


@pytest.mark.parametrize("T", [1 << 24, (1 << 24) + 70001, 80, 700])
def test_long_sums(T):
    """Losses of many like tokens, against 64-bit sums of the probabilities and lse that the call itself
    gives: a tile's at most 128 values are added in fp32 (waves of up to 16, then 8 waves: 24 roundings),
    tiles in 64 bits, a workgroup's sums are rounded to fp32 once and so are lse^2 and the loss: 28
    roundings of 2^-24, however many tokens there are."""
    d, E = 8, 2
    g = torch.Generator().manual_seed(5)
    row, wr = torch.randn(d, generator=g).bfloat16().cuda(), torch.randn(E, d, generator=g).bfloat16().cuda()
    n = row.repeat(T, 1)
    p, lse = torch.empty(T, E, device="cuda"), torch.empty(T, device="cuda")
    sel = torch.tensor([0, 1], dtype=torch.int32, device="cuda").repeat(T, 1)
    sel[: T // 3] = torch.tensor([1, 7], dtype=torch.int32, device="cuda")
    counts, loss = torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    size = lc.lc_moe_balance_scratch_bytes(T, d, E)
    lc.lc_moe_balance_forward(T, d, E, n, wr, sel, p, lse, counts, loss, torch.empty(size, dtype=torch.uint8, device="cuda"),
                              size, lc.LC_BF16, lc.LC_BF16)
    assert counts.tolist() == [T - T // 3, T, T]
    f = counts[:E].double() / (2 * T)
    want = torch.stack([E * (f * p.double().sum(0)).sum() / T, (lse.double() ** 2).sum() / T]).cpu()
    off = (loss.cpu().double() - want).abs() / (28 * 2.0 ** -24 * want)
    assert float(off.max()) <= 1.0, off


@pytest.mark.parametrize("E", [7, 24, 40, 64])
@pytest.mark.parametrize("T", [4097, 8193, 12289, 16385, 20481, 24577, 28673, 33000])
def test_forward_tiles(T, E):
    """Token counts next to each border between the forward's tile heights."""
    d = 72
    s = inputs(T, d, E, "bf16", "bf16", T + E, masked=T % 3 == 0)
    check(call(s, E, "bf16", "bf16", dn="bf16"), reference(s, E, dres=False), d, "bf16")
