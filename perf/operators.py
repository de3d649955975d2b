"""The performance cases of the operators ahead of the sampler: from a decode step's last hidden states to the
logits that are sampled.

  norm    residual addition and root-mean-square norm, the result in the inputs' type and / or in 8 bits
          with a scale per row
  w4      the product of hidden states (bf16, or the norm's 8 bits) with 4-bit weights and group scales:
          the language-model head
  adjust  biases, repetition / frequency / presence penalties and grammar masks on the logits

``own`` false computes them in elementary torch operations in 32 bits; true calls this library.  Calls whose
work is short are made through the prepared objects that a decode loop keeps ("prepared"), the others through
the functions.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_ES = {"bf16": 2, "f32": 4, "i8": 1}
EPS = 1e-5


def _norm(T, D, dtype, wdtype="bf16", residual=True, normed=True, quant=False, prepared=True, name=None):
    c = dict(op="norm", T=T, D=D, dtype=dtype, wdtype=wdtype, residual=residual, normed=normed, quant=quant,
             prepared=prepared)
    if name:
        c["name"] = name
    return c


def _w4(B, N, K, group, x, scales="bf16", zeros=False, out="f32", prepared=True, name=None):
    c = dict(op="w4", B=B, N=N, K=K, group=group, x=x, scales=scales, zeros=zeros, out=out, prepared=prepared)
    if name:
        c["name"] = name
    return c


def _adjust(B, V, dtype, out, H=0, bias=0, mask="none", in_place=False, prepared=True, name=None):
    c = dict(op="adjust", B=B, V=V, dtype=dtype, out=out, H=H, bias=bias, mask=mask, in_place=in_place,
             prepared=prepared)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one sequence's newest token between two layers (latency)
        _norm(1, 4096, "bf16", name="norm_1x4096_bf16"),
        # a decode batch ahead of the 4-bit head: 8 bits with a scale per row, and the residual stream
        _norm(256, 8192, "bf16", normed=False, quant=True, name="norm_256x8192_bf16_8bit"),
        # an odd width in fp32, both outputs, no residual
        _norm(1000, 5121, "f32", wdtype="f32", residual=False, quant=True, name="norm_1000x5121_f32_both"),
        # the tokens of a prompt
        _norm(8192, 4096, "bf16", prepared=False, name="norm_8192x4096_bf16"),
        # one sequence's token through the head (latency and memory)
        _w4(1, 32000, 4096, 128, "bf16", name="w4_1x32000x4096_bf16"),
        # a small odd batch, odd vocabulary, groups of 32 with zero points and fp32 scales
        _w4(13, 100003, 2080, 32, "bf16", scales="f32", zeros=True, name="w4_13x100003x2080_bf16_zeros"),
        # an ordinary decode batch, bf16 hidden states
        _w4(16, 128256, 4096, 128, "bf16", out="bf16", name="w4_16x128256x4096_bf16"),
        # a wide model's decode batch on the norm's 8 bits
        _w4(64, 128256, 8192, 128, "i8", prepared=False, name="w4_64x128256x8192_8bit"),
        # the largest: a full batch of sequences over a wide vocabulary
        _w4(256, 152064, 4096, 128, "i8", prepared=False, name="w4_256x152064x4096_8bit"),
        # a few chat requests with a bias list and a grammar
        _adjust(4, 32000, "f32", "f32", bias=40, mask="few", name="adjust_4x32000_f32_bias_mask"),
        # a decode batch with everything: penalties over 2048 tokens, biases, a grammar on two rows of three
        _adjust(256, 152064, "bf16", "f32", H=2048, bias=300, mask="mixed", prepared=False,
                name="adjust_256x152064_bf16_everything"),
        # structured output: grammar masks alone, in place on fp32 logits
        _adjust(256, 152064, "f32", "f32", mask="mixed", in_place=True, name="adjust_256x152064_f32_in_place"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "w4", "w4", "adjust"])
    if op == "norm":
        D = _log_int(rng, 64, 16384)
        if rng.random() < 0.7:
            D = max(64, D // 64 * 64)
        T = _log_int(rng, 1, min(8192, (8192 * 4096) // D))
        normed, quant = rng.choice([(True, False), (False, True), (True, True)])
        return _norm(T, D, rng.choice(["bf16", "bf16", "f32"]), wdtype=rng.choice(["bf16", "f32"]),
                     residual=rng.random() < 0.7, normed=normed, quant=quant, prepared=T * D < 1 << 24)
    if op == "w4":
        group = rng.choice([32, 64, 128, 128])
        K = max(512, _log_int(rng, 512, 8192) // group * group)
        N = _log_int(rng, 1000, min(256000, 128256 * 8192 // K))
        if rng.random() < 0.5:
            N = max(64, N // 64 * 64)
        B = _log_int(rng, 1, 256)
        B = max(1, min(B, 256 * 152064 * 4096 // (N * K)))
        return _w4(B, N, K, group, rng.choice(["bf16", "i8"]), scales=rng.choice(["bf16", "f32"]),
                   zeros=rng.random() < 0.3, out=rng.choice(["f32", "bf16"]), prepared=rng.random() < 0.5)
    V = _log_int(rng, 1000, 256000)
    if rng.random() < 0.5:
        V = max(64, V // 64 * 64)
    B = _log_int(rng, 1, max(1, min(1024, 256 * 152064 // V)))
    if rng.random() < 0.3:
        dt = rng.choice(["bf16", "f32"])
        return _adjust(B, V, dt, dt, mask=rng.choice(["few", "most", "half", "mixed"]), in_place=True)
    return _adjust(B, V, rng.choice(["bf16", "f32"]), rng.choice(["f32", "f32", "bf16"]),
                   H=rng.choice([0, _log_int(rng, 16, 4096)]), bias=rng.choice([0, min(V // 4, _log_int(rng, 1, 1000))]),
                   mask=rng.choice(["none", "few", "most", "half", "mixed"]), prepared=B * V < 1 << 24)


# --------------------------------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------------------------------
def _gen(seed, what):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 16 + what)
    return g


def _norm_inputs(case, seed):
    T, D, dt = case["T"], case["D"], _DT[case["dtype"]]
    # a layer's output and a residual stream of larger values with a few outlier channels
    x = torch.randn((T, D), generator=_gen(seed, 0), device=DEV)
    big = torch.rand(D, generator=_gen(seed, 1), device=DEV) < 0.005
    chan = 1.0 + 20.0 * big.float()
    s = dict(x=(x * 0.5).to(dt), residual=None)
    if case["residual"]:
        s["residual"] = (torch.randn((T, D), generator=_gen(seed, 2), device=DEV) * 3.0 * chan).to(dt)
    s["weight"] = (0.5 + torch.rand(D, generator=_gen(seed, 3), device=DEV)).to(_DT[case["wdtype"]])
    return s


def _w4_inputs(case, seed):
    B, N, K, G = case["B"], case["N"], case["K"], case["group"]
    s = dict(x_scale=None, zeros=None)
    x = torch.randn((B, K), generator=_gen(seed, 0), device=DEV)
    if case["x"] == "i8":
        s["x"] = torch.clamp(torch.round(x * 32.0), -127, 127).to(torch.int8)
        s["x_scale"] = 0.01 + 0.04 * torch.rand(B, generator=_gen(seed, 1), device=DEV)
    else:
        s["x"] = x.to(torch.bfloat16)
    g = _gen(seed, 2)
    packed = torch.empty((N, K // 2), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 28) // K)
    for lo in range(0, N, step):  # bell-shaped weights, two to a byte, the even column in the low bits
        n = min(N, lo + step) - lo
        q = torch.clamp(torch.round(torch.randn((n, K), generator=g, device=DEV) * 2.7 + 8.0), 0, 15).to(torch.uint8)
        packed[lo:lo + n] = q[:, 0::2] | (q[:, 1::2] << 4)
    s["packed"] = packed
    s["scales"] = (0.004 + 0.008 * torch.rand((N, K // G), generator=_gen(seed, 3), device=DEV)).to(_DT[case["scales"]])
    if case["zeros"]:
        s["zeros"] = torch.randint(5, 12, (N, K // G), generator=_gen(seed, 4), device=DEV, dtype=torch.uint8)
    return s


def _adjust_inputs(case, seed):
    B, V, H, nb, kind = case["B"], case["V"], case["H"], case["bias"], case["mask"]
    s = dict(hist_ids=None, bias_ids=None, mask=None, mask_index=None)
    # language-model-like logits: noise with Zipf-ranked offsets
    rank = torch.empty(V, dtype=torch.float32, device=DEV)
    perm = torch.randperm(V, generator=_gen(seed, 1), device=DEV)
    rank[perm] = torch.arange(1, V + 1, dtype=torch.float32, device=DEV)
    off = -1.1 * torch.log(rank)
    logits = torch.empty((B, V), dtype=_DT[case["dtype"]], device=DEV)
    g = _gen(seed, 0)
    step = max(1, (1 << 25) // V)
    for lo in range(0, B, step):
        n = min(B, lo + step) - lo
        logits[lo:lo + n] = (torch.randn((n, V), generator=g, device=DEV) * 3.0 + off).to(logits.dtype)
    s["logits"] = logits
    if H:  # H tokens a row, ranks with probability proportional to r^-1.2
        w = torch.cumsum(torch.arange(1, V + 1, dtype=torch.float64, device=DEV) ** -1.2, 0)
        u = torch.rand(B * H, dtype=torch.float64, generator=_gen(seed, 2), device=DEV) * w[-1]
        s["hist_ids"] = perm[torch.searchsorted(w, u).clamp_(max=V - 1)].to(torch.int32)
        s["hist_offsets"] = torch.arange(B + 1, dtype=torch.int64, device=DEV) * H
        gp = _gen(seed, 3)
        s["rep"] = 1.0 + 0.3 * torch.rand(B, generator=gp, device=DEV)
        s["freq"] = 0.4 * torch.rand(B, generator=gp, device=DEV)
        s["pres"] = 0.4 * torch.rand(B, generator=gp, device=DEV)
    if nb:  # nb distinct ids a row: a stride walk through the permuted vocabulary from a row's own start
        start = torch.randint(0, V, (B, 1), generator=_gen(seed, 4), device=DEV)
        at = (start + torch.arange(nb, device=DEV) * max(1, V // nb)) % V
        s["bias_ids"] = perm[at].to(torch.int32).reshape(-1).contiguous()
        val = torch.randn(B * nb, generator=_gen(seed, 5), device=DEV) * 5.0
        # some entries ban their token with the usual -100, some outright
        u = torch.rand(B * nb, generator=_gen(seed, 6), device=DEV)
        val = torch.where(u < 0.2, torch.full_like(val, -100.0), val)
        s["bias_values"] = torch.where(u > 0.98, torch.full_like(val, -math.inf), val)
        s["bias_offsets"] = torch.arange(B + 1, dtype=torch.int64, device=DEV) * nb
    if kind != "none":
        M = (B + 1) // 2 if kind == "mixed" else B  # "mixed": rows share grammar states, a third has none
        W = (V + 31) // 32
        words = torch.empty((M, W), dtype=torch.int32, device=DEV)
        gm = _gen(seed, 7)
        share = {"few": 0.0005, "most": 0.99, "half": 0.5}
        for lo in range(0, M, 64):
            n = min(M, lo + 64) - lo
            p = torch.tensor([share[kind] if kind != "mixed" else share[("few", "few", "most", "half")[(lo + i) % 4]]
                              for i in range(n)], device=DEV)
            bits = torch.rand((n, W * 32), generator=gm, device=DEV) < p[:, None]
            sh = torch.arange(32, dtype=torch.int64, device=DEV)
            word = (bits.view(n, W, 32).to(torch.int64) << sh).sum(2)
            words[lo:lo + n] = torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)
        s["mask"] = words
        if kind == "mixed":
            i = torch.arange(B, device=DEV)
            s["mask_index"] = torch.where(i % 3 == 2, torch.full_like(i, -1), i % M).to(torch.int32)
    return s


def _own_call(case, s):
    """The library's objects of this case's inputs: weight handle, parameters, output buffers and, for the
    short calls, the prepared call."""
    import paper_2606_01927_amd as alb

    if case["op"] == "norm":
        T, D = case["T"], case["D"]
        kw = dict(eps=EPS, residual=s["residual"], normed=case["normed"], quant=case["quant"])
        if not case["prepared"]:
            return lambda: alb.rms_norm(s["x"], s["weight"], **kw)
        out = alb.NormOut(
            y=torch.empty((T, D), dtype=s["x"].dtype, device=DEV) if case["normed"] else None,
            residual=torch.empty_like(s["x"]) if case["residual"] else None,
            q=torch.empty((T, D), dtype=torch.int8, device=DEV) if case["quant"] else None,
            scale=torch.empty(T, dtype=torch.float32, device=DEV) if case["quant"] else None)
        return alb.PreparedNorm(s["x"], s["weight"], out=out, **kw)
    if case["op"] == "w4":
        w = alb.W4Weight(s["packed"], s["scales"], s["zeros"])
        dt = _DT[case["out"]]
        if not case["prepared"]:
            return lambda: alb.matmul_w4(s["x"], w, x_scale=s["x_scale"], out_dtype=dt)
        out = torch.empty((case["B"], case["N"]), dtype=dt, device=DEV)
        return alb.PreparedMatmulW4(s["x"], w, x_scale=s["x_scale"], out=out)
    prm = None
    if case["H"]:
        prm = alb.SamplingParams(repetition_penalty=s["rep"], frequency_penalty=s["freq"], presence_penalty=s["pres"],
                                 hist_offsets=s["hist_offsets"], hist_ids=s["hist_ids"])
    con = alb.Constraints(mask=s["mask"], mask_index=s["mask_index"])
    if case["bias"]:
        con.bias_offsets, con.bias_ids, con.bias_values = s["bias_offsets"], s["bias_ids"], s["bias_values"]
    if not case["prepared"]:
        return lambda: alb.adjust_logits(s["logits"], prm, con, out=s["logits"] if case["in_place"] else None,
                                         out_dtype=_DT[case["out"]])
    out = s["logits"] if case["in_place"] else torch.empty((case["B"], case["V"]), dtype=_DT[case["out"]], device=DEV)
    return alb.PreparedAdjust(s["logits"], prm, con, out=out)


_INPUTS = {"norm": _norm_inputs, "w4": _w4_inputs, "adjust": _adjust_inputs}


def prepare(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    s["case"] = case
    if own:
        s["call"] = _own_call(case, s)
    return s


# --------------------------------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if own:
        r = state["call"]()
        if case["op"] == "norm":
            return _norm_result(case, r.y, r.residual, r.q, r.scale)
        return [r] if case["op"] == "w4" else [r[0], r[1]]
    return {"norm": _plain_norm, "w4": _plain_w4, "adjust": _plain_adjust}[case["op"]](case, state)


def _norm_result(case, y, residual, q, scale):
    """The outputs a case asked for.  The 8-bit values and their scales are the output as a program holds it."""
    r = []
    if case["residual"]:
        r.append(residual)
    if case["normed"]:
        r.append(y)
    if case["quant"]:
        r += [q.float() * scale[:, None], scale]
    return r


def _plain_norm(case, s):
    h = s["x"].float()
    res = None
    if s["residual"] is not None:
        h = h + s["residual"].float()
        res = h.to(s["x"].dtype)
    y = h * (1.0 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + EPS)) * s["weight"].float()
    q = scale = None
    if case["quant"]:
        amax = y.abs().amax(dim=1)
        scale = amax / 127.0
        q = torch.round(y * (127.0 / amax)[:, None])
    return _norm_result(case, y.to(s["x"].dtype), res, q, scale)


def _plain_w4(case, s):
    N, K, G = case["N"], case["K"], case["group"]
    p = s["packed"]
    w = torch.stack((p & 15, p >> 4), dim=2).view(N, K // G, G).float()
    w = w - (8.0 if s["zeros"] is None else s["zeros"].float()[:, :, None])
    w = (w * s["scales"].float()[:, :, None]).view(N, K)
    out = s["x"].float() @ w.t()
    if s["x_scale"] is not None:
        out = out * s["x_scale"][:, None]
    return [out.to(_DT[case["out"]])]


def _allowed(case, s):
    V = case["V"]
    v = torch.arange(V, device=DEV)
    m = s["mask"] if s["mask_index"] is None else s["mask"][s["mask_index"].clamp(min=0).long()]
    bit = (m[:, v >> 5] >> (v & 31).to(torch.int32)) & 1
    ok = bit != 0
    return ok if s["mask_index"] is None else ok | (s["mask_index"] < 0)[:, None]


def _plain_adjust(case, s):
    B, V = case["B"], case["V"]
    flags = torch.zeros(B, dtype=torch.int32, device=DEV)
    if case["in_place"]:
        s["logits"].masked_fill_(~_allowed(case, s), -math.inf)
        return [s["logits"], flags]
    x = s["logits"].float()
    rows = torch.arange(B, device=DEV)[:, None]
    if case["bias"]:
        ids = s["bias_ids"].view(B, -1).long()
        x[rows, ids] = x[rows, ids] + s["bias_values"].view(B, -1)
    if case["H"]:
        ids = s["hist_ids"].view(B, -1).long()
        cnt = torch.zeros((B, V), dtype=torch.float32, device=DEV)
        cnt.scatter_add_(1, ids, torch.ones(ids.shape, device=DEV))
        seen = cnt > 0
        rep, freq, pres = s["rep"][:, None], s["freq"][:, None], s["pres"][:, None]
        pen = torch.where(x > 0, x / rep, x * rep) - freq * cnt - pres
        x = torch.where(seen, pen, x)
    if s["mask"] is not None:
        x = x.masked_fill(~_allowed(case, s), -math.inf)
    return [x.to(_DT[case["out"]]), flags]


# --------------------------------------------------------------------------------------------------
# What a pass cannot do without, and the results from the definitions in 64 bits
# --------------------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "norm":
        T, D, es = case["T"], case["D"], _ES[case["dtype"]]
        each = es * (1 + 2 * case["residual"] + case["normed"]) + case["quant"]
        return {"bytes": T * D * each + D * _ES[case["wdtype"]] + (4 * T if case["quant"] else 0),
                "flops": T * D * (5 + 2 * case["quant"])}
    if case["op"] == "w4":
        B, N, K, G = case["B"], case["N"], case["K"], case["group"]
        per_group = _ES[case["scales"]] + (1 if case["zeros"] else 0)
        return {"bytes": N * K // 2 + N * (K // G) * per_group + B * K * _ES["i8" if case["x"] == "i8" else "bf16"]
                + (4 * B if case["x"] == "i8" else 0) + B * N * _ES[case["out"]], "flops": 2 * B * N * K}
    B, V, kind = case["B"], case["V"], case["mask"]
    rows = {"none": 0.0, "mixed": 2.0 / 3.0}.get(kind, 1.0) * B
    if case["in_place"]:  # the mask's bits, and the masked logits' places
        gone = {"few": 0.9995, "most": 0.01, "half": 0.5, "mixed": (2 * 0.9995 + 0.01 + 0.5) / 4}[kind]
        return {"bytes": int(rows * (V / 8 + gone * V * _ES[case["dtype"]])), "flops": 0}
    return {"bytes": int(B * V * (_ES[case["dtype"]] + _ES[case["out"]]) + rows * V / 8
                         + 8 * B * case["bias"] + 4 * B * case["H"]),
            "flops": B * (4 * case["H"] + case["bias"])}


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h += s["residual"].double()
        rms = torch.linalg.vector_norm(h, dim=1).square_().div_(case["D"]).add_(EPS).sqrt_()
        y = h / rms[:, None] * s["weight"].double()
        r = [h] if case["residual"] else []
        if case["normed"]:
            r.append(y)
        if case["quant"]:
            step = y.abs().amax(dim=1) / 127.0
            r += [torch.round(y / step[:, None]) * step[:, None], step]
        return r
    if case["op"] == "w4":
        N, K, G = case["N"], case["K"], case["group"]
        x = s["x"].double()
        if s["x_scale"] is not None:
            x = x * s["x_scale"].double()[:, None]
        out = torch.empty((case["B"], N), dtype=torch.float64, device=DEV)
        for lo in range(0, N, 8192):
            p = s["packed"][lo:lo + 8192]
            w = torch.empty((p.shape[0], K), dtype=torch.float64, device=DEV)
            w[:, 0::2] = (p % 16).double()
            w[:, 1::2] = torch.div(p, 16, rounding_mode="floor").double()
            z = torch.full((1, 1), 8.0, dtype=torch.float64, device=DEV) if s["zeros"] is None else \
                s["zeros"][lo:lo + 8192].double().repeat_interleave(G, dim=1)
            w = (w - z) * s["scales"][lo:lo + 8192].double().repeat_interleave(G, dim=1)
            out[:, lo:lo + 8192] = torch.mm(x, w.t())
        return [out]
    B, V = case["B"], case["V"]
    x = s["logits"].double()
    for i in range(B):
        if case["bias"]:
            at = slice(i * case["bias"], (i + 1) * case["bias"])
            x[i].index_add_(0, s["bias_ids"][at].long(), s["bias_values"][at].double())
        if case["H"]:
            ids, n = torch.unique(s["hist_ids"][i * case["H"]:(i + 1) * case["H"]].long(), return_counts=True)
            v = x[i, ids]
            rep, freq, pres = s["rep"][i].double(), s["freq"][i].double(), s["pres"][i].double()
            x[i, ids] = torch.where(v > 0, v / rep, v * rep) - n.double() * freq - pres
        if s["mask"] is not None:
            m = i if s["mask_index"] is None else int(s["mask_index"][i])
            if m >= 0:
                bits = torch.bitwise_and(s["mask"][m][:, None], torch.bitwise_left_shift(
                    torch.ones(32, dtype=torch.int32, device=DEV), torch.arange(32, dtype=torch.int32, device=DEV)))
                x[i][bits.view(-1)[:V] == 0] = -math.inf
    return [x, None]
