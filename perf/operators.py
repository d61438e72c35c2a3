"""Performance cases of the operators a layer of an 8-bit floating point (e4m3) checkpoint with normed heads runs, one
call each, over the sizes a serving program meets.

Kinds of case

  quant  k_quant_f8: rows of activations to e4m3 with one fp32 scale per row and 128 columns
  gemm   k_gemm_f8: rows times an e4m3 matrix with one fp32 scale per 128 x 128 block; the rows come quantised ("f8") or as
         fp32 / bf16 rows, which the call quantises itself
  norm   k_qk_norm_rope: RMS norm of every query and key head and its rotation, read out of the fused QKV rows

Widths are those of synth.configs (1B-, 7B-, 8B- and 13B-shaped models) and odd ones next to them.  In the plain form
every operator is written with elementary torch operations in 32 bits and rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
LEAST = 2.0 ** -96      # a group's largest magnitude counts as at least this
WORKSPACE = 32 << 20    # scratch a serving program keeps for partial results, beside the quantised rows
EPS = 1e-5

TYPES = {"f8": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token through the output projection of the 1B-shaped draft: the smallest call, latency
        {"name": "gemm-1b-token", "kind": "gemm", "R": 1, "N": 2048, "K": 2048, "x": "f32", "y": "f32"},
        # one token through the gate / up projections of the 8B-shaped target: a stream of the weights
        {"name": "gemm-8b-token-gate-up", "kind": "gemm", "R": 1, "N": 28672, "K": 4096, "x": "bf16", "y": "f32"},
        # verification of eight drafted tokens, down projection of the 13B-shaped target
        {"name": "gemm-13b-verify-down", "kind": "gemm", "R": 9, "N": 5120, "K": 13824, "x": "f8", "y": "f32"},
        # verification of many sequences, an uneven number of rows, down projection of the 7B-shaped target
        {"name": "gemm-7b-batch-verify", "kind": "gemm", "R": 137, "N": 4096, "K": 11008, "x": "bf16", "y": "bf16"},
        # odd sizes: a last block of 16 columns, a width that no tile divides
        {"name": "gemm-odd", "kind": "gemm", "R": 37, "N": 777, "K": 1040, "x": "f8", "y": "bf16"},
        # one prompt through the fused QKV projection of the 8B-shaped target
        {"name": "gemm-8b-prompt-qkv", "kind": "gemm", "R": 1024, "N": 6144, "K": 4096, "x": "f32", "y": "f32"},
        # four long prompts through its gate / up projections: the largest product
        {"name": "gemm-8b-prompts-gate-up", "kind": "gemm", "R": 4096, "N": 28672, "K": 4096, "x": "f8", "y": "bf16"},
        # rows of one verification step
        {"name": "quant-rows", "kind": "quant", "R": 9, "K": 5120, "x": "f32"},
        # activations of the MLP for four long prompts
        {"name": "quant-prompts", "kind": "quant", "R": 4096, "K": 14336, "x": "bf16"},
        # one token of the 8B-shaped target
        {"name": "norm-8b-token", "kind": "norm", "R": 1, "nq": 32, "nkv": 8, "hd": 128, "x": "f32", "y": "f32", "pad": 0.0},
        # many sequences through the small draft, a few rows of padding among them
        {"name": "norm-draft-batch", "kind": "norm", "R": 131, "nq": 12, "nkv": 12, "hd": 64, "x": "f32", "y": "bf16", "pad": 0.1},
        # long prompts of the 8B-shaped target
        {"name": "norm-8b-prompts", "kind": "norm", "R": 16384, "nq": 32, "nkv": 8, "hd": 128, "x": "bf16", "y": "bf16", "pad": 0.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "gemm", "quant", "norm", "norm"])
    if kind == "gemm":
        K = 16 * _log_int(rng, 8, 896)
        N = _log_int(rng, 64, 28672)
        R = min(_log_int(rng, 1, 4096), max(1, int(4096 * 28672 * 4096 / (N * K))))
        return {"kind": kind, "R": R, "N": N, "K": K, "x": rng.choice(["f8", "f32", "bf16"]), "y": rng.choice(["f32", "bf16"])}
    if kind == "quant":
        return {"kind": kind, "R": _log_int(rng, 1, 4096), "K": 16 * _log_int(rng, 4, 896), "x": rng.choice(["f32", "bf16"])}
    nq, nkv = rng.choice([(4, 4), (8, 2), (12, 12), (32, 8), (40, 40), (7, 1), (20, 5)])
    return {"kind": kind, "R": min(_log_int(rng, 1, 16384), 16384 * 40 // (nq + nkv)), "nq": nq, "nkv": nkv,
            "hd": rng.choice([32, 64, 80, 96, 128]), "x": rng.choice(["f32", "bf16"]), "y": rng.choice(["f32", "bf16"]),
            "pad": rng.choice([0.0, 0.1, 0.3])}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _activations(gen, R, K):
    """Rows as a model's layers see them: a few columns are much larger than the others, and rows differ in size."""
    cols = torch.exp(0.5 * torch.randn(K, generator=gen, device="cuda"))
    cols[torch.randint(0, K, (max(1, K // 100),), generator=gen, device="cuda")] *= 12.0
    rows = torch.exp(0.3 * torch.randn((R, 1), generator=gen, device="cuda"))
    return torch.randn((R, K), generator=gen, device="cuda") * cols * rows


def _quantise(x):
    """Plain form of the quantiser: x fp32 [R][K] -> e4m3 [R][K], scale [blocks][R]."""
    R, K = x.shape
    KB = _blocks(K)
    g = torch.nn.functional.pad(x, (0, KB * BLOCK - K)).reshape(R, KB, BLOCK)
    a = g.abs().amax(dim=2).clamp_min(LEAST)
    top = torch.full_like(a, E4M3_MAX)
    q = (g * (top / a)[:, :, None]).reshape(R, KB * BLOCK)[:, :K].to(torch.float8_e4m3fn)
    return q.contiguous(), (a / top).t().contiguous()


def _spread(s, n):
    """One value per block of the last axis -> one per element."""
    return s.repeat_interleave(BLOCK, dim=-1)[..., :n]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, R = case["kind"], case["R"]
    st = {"case": case}
    if kind == "norm":
        nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
        tx, ty = TYPES[case["x"]], TYPES[case["y"]]
        n_pos = 4096
        # the fused product's rows: query heads, key heads, then the value heads, which stay as they are
        qkv = (torch.randn((R, (nq + 2 * nkv) * hd), generator=gen, device="cuda") *
               torch.exp(0.5 * torch.randn((R, 1), generator=gen, device="cuda"))).to(tx)
        st["q"] = qkv[:, : nq * hd].unflatten(1, (nq, hd))
        st["k"] = qkv[:, nq * hd: (nq + nkv) * hd].unflatten(1, (nkv, hd))
        st["q_norm"] = 1.0 + 0.2 * torch.randn(hd, generator=gen, device="cuda")
        st["k_norm"] = 1.0 + 0.2 * torch.randn(hd, generator=gen, device="cuda")
        ang = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * \
            500000.0 ** (-2.0 * torch.arange(hd // 2, device="cuda", dtype=torch.float64) / hd)[None, :]
        st["cos"], st["sin"] = torch.cos(ang).float(), torch.sin(ang).float()
        pos = torch.randint(0, n_pos, (R,), generator=gen, device="cuda", dtype=torch.int32)
        if case["pad"]:  # rows without a position are padding
            pos[torch.rand(R, generator=gen, device="cuda") < case["pad"]] = -1
        st["pos"] = pos
        st["q_out"] = torch.zeros((R, nq, hd), dtype=ty, device="cuda")
        st["k_out"] = torch.zeros((R, nkv, hd), dtype=ty, device="cuda")
        return st
    K = case["K"]
    x = _activations(gen, R, K)
    if kind == "quant":
        st["x"] = x.to(TYPES[case["x"]])
        st["q"] = torch.zeros((R, K), dtype=torch.float8_e4m3fn, device="cuda")
        st["scale"] = torch.zeros((_blocks(K), R), dtype=torch.float32, device="cuda")
        return st
    N = case["N"]
    KB, NB = _blocks(K), _blocks(N)
    # a checkpoint's matrix: normal values, one scale per 128 x 128 block that takes the block's largest to 448
    w = 0.02 * torch.randn((NB * BLOCK, KB * BLOCK), generator=gen, device="cuda").reshape(NB, BLOCK, KB, BLOCK)
    ws = w.abs().amax(dim=(1, 3)) / E4M3_MAX
    st["w"] = (w / ws[:, None, :, None]).reshape(NB * BLOCK, KB * BLOCK)[:N, :K].to(torch.float8_e4m3fn).contiguous()
    st["w_scale"] = ws.contiguous()
    if case["x"] == "f8":
        st["x"], st["x_scale"] = _quantise(x)
    else:
        st["x"], st["x_scale"] = x.to(TYPES[case["x"]]), None
    st["y"] = torch.zeros((R, N), dtype=TYPES[case["y"]], device="cuda")
    st["workspace"] = torch.empty(132 * R * KB + WORKSPACE, dtype=torch.uint8, device="cuda")
    return st


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2504_00030_amd as pk
        stream = torch.cuda.current_stream().cuda_stream
        if kind == "quant":
            pk.k_quant_f8(state["x"], state["q"], state["scale"], stream=stream)
            return {"q": state["q"], "scale": state["scale"]}
        if kind == "gemm":
            pk.k_gemm_f8(state["w"], state["w_scale"], state["x"], state["y"], x_scale=state["x_scale"],
                         workspace=state["workspace"], stream=stream)
            return {"y": state["y"]}
        pk.k_qk_norm_rope(state["q"], state["k"], state["q_norm"], state["k_norm"], state["cos"], state["sin"], state["pos"],
                          state["q_out"], state["k_out"], eps=EPS, stream=stream)
        return {"q": state["q_out"], "k": state["k_out"]}
    if kind == "quant":
        q, scale = _quantise(state["x"].float())
        return {"q": q, "scale": scale}
    if kind == "gemm":
        x, xs, w = state["x"], state["x_scale"], state["w"]
        N, K = w.shape
        if xs is None:
            x, xs = _quantise(x.float())
        wf = w.float() * _spread(_spread(state["w_scale"], K).t(), N).t()
        return {"y": ((x.float() * _spread(xs.t(), K)) @ wf.t()).to(state["y"].dtype)}
    pos, hd = state["pos"], state["case"]["hd"]
    half, n_pos = hd // 2, state["cos"].shape[0]
    valid = ((pos >= 0) & (pos < n_pos))[:, None, None]
    at = pos.clamp(0, n_pos - 1).long()
    c, s = state["cos"][at][:, None, :], state["sin"][at][:, None, :]
    out = {}
    for name in ("q", "k"):
        h = state[name].float()
        h = h * torch.rsqrt((h * h).mean(dim=2, keepdim=True) + EPS) * state[name + "_norm"]
        a, b = h[..., :half], h[..., half:]
        r = torch.cat([a * c - b * s, b * c + a * s], dim=2).to(state[name + "_out"].dtype)
        out[name] = torch.where(valid, r, state[name + "_out"])
    return out


def work(case):
    R = case["R"]
    size = {"f8": 1.0, "bf16": 2.0, "f32": 4.0}
    if case["kind"] == "norm":
        rows = R * (1.0 - case["pad"])
        n = rows * (case["nq"] + case["nkv"]) * case["hd"]
        tables = min(rows, 4096.0) * case["hd"] * 4.0
        return {"bytes": n * (size[case["x"]] + size[case["y"]]) + tables + 4.0 * R, "flops": 8.0 * n}
    K, KB = case["K"], _blocks(case["K"])
    if case["kind"] == "quant":
        return {"bytes": R * K * (size[case["x"]] + 1.0) + 4.0 * R * KB, "flops": 3.0 * R * K}
    N = case["N"]
    b = N * K + 4.0 * _blocks(N) * KB + R * K * size[case["x"]] + R * N * size[case["y"]]
    return {"bytes": b + (4.0 * R * KB if case["x"] == "f8" else 0.0), "flops": 2.0 * R * N * K}


def _e4m3(v):
    """The nearest e4m3 value (ties to the even one) of 64-bit values of magnitude up to 448, by its definition: steps of
    2^-3 of the power of two below, never finer than 2^-9."""
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -40)))
    e = torch.where(torch.exp2(e) > v.abs(), e - 1, e)
    e = torch.where(torch.exp2(e + 1) <= v.abs(), e + 1, e)
    step = torch.exp2(e.clamp_min(-6.0) - 3.0)
    return torch.round(v / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        pos, half = st["pos"].long(), case["hd"] // 2
        res = {}
        for name in ("q", "k"):
            h, o = st[name].double(), st[name + "_out"].double()
            norm = torch.sqrt(torch.sum(h ** 2, dim=2, keepdim=True) / case["hd"] + EPS)
            h = h / norm * st[name + "_norm"].double()
            for rows in torch.nonzero(pos >= 0).flatten().split(4096):
                c, s = st["cos"].double()[pos[rows]].unsqueeze(1), st["sin"].double()[pos[rows]].unsqueeze(1)
                z = torch.complex(h[rows, :, :half], h[rows, :, half:]) * torch.complex(c, s)
                o[rows, :, :half], o[rows, :, half:] = z.real, z.imag
            res[name] = o
        return res
    x, K = st["x"], case["K"]
    if kind == "quant" or case["x"] != "f8":
        # the definition rounds the scale, the factor and the scaled value to 32 bits before the rounding to e4m3
        q, scales = torch.zeros(x.shape, dtype=torch.float64, device="cuda"), []
        for k0 in range(0, K, BLOCK):
            part = x[:, k0: k0 + BLOCK].double()
            a = part.abs().max(dim=1).values.clamp_min(LEAST)
            factor = (E4M3_MAX / a).float().double()
            q[:, k0: k0 + BLOCK] = _e4m3((part * factor[:, None]).float().double())
            scales.append((a / E4M3_MAX).float().double())
        scale = torch.stack(scales)
    else:
        q, scale = x.double(), st["x_scale"].double()
    if kind == "quant":
        return {"q": q, "scale": scale}
    y = torch.zeros((case["R"], case["N"]), dtype=torch.float64, device="cuda")
    for b, k0 in enumerate(range(0, K, BLOCK)):
        t = q[:, k0: k0 + BLOCK] @ st["w"][:, k0: k0 + BLOCK].double().t().contiguous()
        for n0 in range(0, case["N"], BLOCK):
            t[:, n0: n0 + BLOCK] *= st["w_scale"][n0 // BLOCK, b].double()
        y += t * scale[b][:, None]
    return {"y": y}
