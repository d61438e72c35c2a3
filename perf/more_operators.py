"""Performance cases of the operators of one verification pass over a batch of sequences that begin alike, one call each:
rotary tables, rotation with the writes of the paged cache, attention over a shared prefix and the sequences' own positions,
and the verification of the drafted tokens against given random numbers.

Kinds of case

  tables  k_rope_tables: cosines and sines of every position, with the scalings for long contexts
  rope    k_rope_cache: rotation of query and key heads (half or interleaved pairs, the whole head or its first part),
          queries to rows, keys and values to pages
  attn    k_attn_shared: every row attends to one prefix that all sequences share and to its own sequence's positions
  verify  k_verify: accepted drafts and the next token from the two models' probabilities and given uniforms

Head layouts and vocabularies are those of synth.configs (tiny, 1B-, 7B-, 8B- and 13B-shaped models) and odd ones next to
them.  In the plain form every operator is written with elementary torch operations in 32 bits (angles, the sums of the draw
and the accept test in 64) and rounded once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2.0, "f32": 4.0}


def listed():
    return [
        # tables of the tiny pair's heads for a short context: the smallest call, latency
        {"name": "tables-short", "kind": "tables", "n_pos": 512, "rot": 32, "scaling": "plain"},
        # 128-element heads over a context stretched from 32768 to 131072 positions
        {"name": "tables-long-ramp", "kind": "tables", "n_pos": 131072, "rot": 128, "scaling": "ramp"},
        # one token of the 8B-shaped target, fp32 projections into a bf16 cache
        {"name": "rope-8b-token", "kind": "rope", "R": 1, "nq": 32, "nkv": 8, "hd": 128, "rot": 128, "inter": False,
         "x": "f32", "y": "bf16", "page": 64, "pad": 0.0},
        # verification rows of many sequences through the small draft: interleaved pairs, half of the head, some padding
        {"name": "rope-draft-batch", "kind": "rope", "R": 131, "nq": 12, "nkv": 12, "hd": 64, "rot": 32, "inter": True,
         "x": "bf16", "y": "bf16", "page": 16, "pad": 0.1},
        # long prompts of the 8B-shaped target
        {"name": "rope-8b-prompts", "kind": "rope", "R": 16384, "nq": 32, "nkv": 8, "hd": 128, "rot": 128, "inter": False,
         "x": "bf16", "y": "bf16", "page": 64, "pad": 0.0},
        # one sequence, one token of the 1B-shaped model behind a short prefix: the smallest attention, latency
        {"name": "attn-1b-token", "kind": "attn", "B": 1, "rows": 1, "ragged": False, "nq": 32, "nkv": 8, "hd": 64, "t": "bf16",
         "prefix": 256, "own": 100, "page": 64},
        # verification of the tiny fp32 pair, uneven sequences, a prefix that ends inside a page
        {"name": "attn-tiny-verify", "kind": "attn", "B": 5, "rows": 9, "ragged": True, "nq": 4, "nkv": 4, "hd": 32, "t": "f32",
         "prefix": 77, "own": 90, "page": 16},
        # verification of 13B-shaped sequences (no shared heads), long own parts of uneven length: a stream of the caches
        {"name": "attn-13b-verify", "kind": "attn", "B": 8, "rows": 5, "ragged": True, "nq": 40, "nkv": 40, "hd": 128, "t": "bf16",
         "prefix": 2001, "own": 4096, "page": 64},
        # verification of 64 sequences of the 8B-shaped target behind one long document
        {"name": "attn-8b-verify", "kind": "attn", "B": 64, "rows": 9, "ragged": True, "nq": 32, "nkv": 8, "hd": 128, "t": "bf16",
         "prefix": 8192, "own": 700, "page": 64},
        # questions of 256 tokens each put to that document: prompts, the largest product of rows and positions
        {"name": "attn-8b-prompts", "kind": "attn", "B": 8, "rows": 256, "ragged": False, "nq": 32, "nkv": 8, "hd": 128, "t": "bf16",
         "prefix": 8192, "own": 256, "page": 64},
        # one sequence of the 7B-shaped pair, four drafts, fp32 probabilities
        {"name": "verify-7b", "kind": "verify", "B": 1, "k": 4, "ragged": False, "vocab": 32000, "t": "f32", "q": True, "top": False},
        # 64 sequences of the 8B-shaped pair, up to eight drafts each, small probabilities filtered out
        {"name": "verify-8b-batch", "kind": "verify", "B": 64, "k": 8, "ragged": True, "vocab": 128256, "t": "f32", "q": True, "top": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "rope", "rope", "attn", "attn", "attn", "verify", "verify"])
    if kind == "tables":
        rot = 2 * _log_int(rng, 8, 64)
        return {"kind": kind, "n_pos": _log_int(rng, 300, 131072), "rot": rot, "scaling": rng.choice(["plain", "linear", "base", "bands", "ramp"])}
    if kind == "rope":
        nq, nkv = rng.choice([(4, 4), (8, 2), (12, 12), (32, 8), (40, 40), (7, 1), (20, 5)])
        hd = rng.choice([32, 64, 80, 96, 128])
        return {"kind": kind, "R": min(_log_int(rng, 1, 16384), 8192 * 48 // (nq + 2 * nkv)), "nq": nq, "nkv": nkv, "hd": hd,
                "rot": rng.choice([hd, hd, hd // 2, hd // 4 * 2 - 2]), "inter": rng.random() < 0.5, "x": rng.choice(["f32", "bf16"]),
                "y": rng.choice(["f32", "bf16"]), "page": rng.choice([16, 64, 128]), "pad": rng.choice([0.0, 0.1, 0.3])}
    if kind == "verify":
        vocab = _log_int(rng, 500, 128256)
        return {"kind": kind, "B": _log_int(rng, 1, 64), "k": rng.randint(1, 8), "ragged": rng.random() < 0.5, "vocab": vocab,
                "t": rng.choice(["f32", "f32", "bf16"]), "q": rng.random() < 0.75, "top": rng.random() < 0.5}
    t = rng.choice(["bf16", "bf16", "bf16", "f32"])
    nq, nkv = rng.choice([(4, 4), (8, 2), (12, 12), (32, 8), (40, 40), (7, 1), (20, 5)])
    hd = rng.choice([32, 64, 80, 96, 128])
    B = _log_int(rng, 1, 64)
    rows = _log_int(rng, 1, 256)
    while B * rows > (2048 if t == "bf16" else 256):
        rows = max(1, rows // 2)
    prefix, own_len = rng.choice([0, 1, 1, 1]) * _log_int(rng, 1, 8192), max(rows, _log_int(rng, 1, 4096))
    while B * own_len * nkv > (8 * 4096 * 20 if t == "bf16" else 8 * 4096 * 5):
        own_len = max(rows, own_len // 2)
        if own_len == rows:
            break
    most = 2048 * 32 * 8320 * 128
    while B * rows * nq * (prefix + own_len) * hd > (most if t == "bf16" else most // 16):
        prefix //= 2
        if prefix == 0:
            break
    return {"kind": kind, "B": B, "rows": rows, "ragged": rng.random() < 0.6, "nq": nq, "nkv": nkv, "hd": hd, "t": t, "prefix": prefix,
            "own": own_len, "page": rng.choice([8, 16, 32, 64, 128])}


def _lengths(case):
    """Rows and own positions of every sequence of an attention case (the rows are the last of the positions)."""
    if not case["ragged"]:
        return [case["rows"]] * case["B"], [max(case["own"], case["rows"])] * case["B"]
    rows = [1 + (7919 * b + 3) % case["rows"] for b in range(case["B"])]
    return rows, [r + int((0.618034 * (b + 1) % 1.0) * max(0, case["own"] - r)) for b, r in enumerate(rows)]


def _drafts(case):
    if not case["ragged"]:
        return [case["k"]] * case["B"]
    return [(5 * b + 2) % (case["k"] + 1) for b in range(case["B"])]


def _starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


SCALED = {  # arguments of the scalings, as a model's configuration states them
    "plain": {},
    "linear": {"factor": 4.0},
    "base": {"factor": 4.0},
    "bands": {"factor": 8.0, "low": 1.0, "high": 4.0, "context": 8192.0},
    "ramp": {"factor": 4.0, "low": 1.0, "high": 32.0, "context": 32768.0},
}
THETA = 500000.0


def _probabilities(gen, rows, vocab, near=None):
    """Log weights that fall with a token's rank, another order in every row; `near` gives rows a draft approximates."""
    if near is None:
        a = next(a for a in range(int(0.381966 * vocab), 2 * vocab) if math.gcd(a, vocab) == 1)
        off = torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda")
        near = -1.2 * torch.log1p(((torch.arange(vocab, device="cuda") * a)[None, :] + off).remainder_(vocab).float())
    return near + 0.6 * torch.randn((rows, vocab), generator=gen, device="cuda")


def _filtered(logits, top, dtype):
    e = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    if top:
        e = torch.where(e < 1e-3, torch.zeros_like(e), e)
    return (e / e.sum(dim=1, keepdim=True)).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    st = {"case": case}
    if kind == "tables":
        half = case["rot"] // 2
        # another seed is another base near the usual one: the inputs of this call are numbers
        st["theta"] = THETA * (1.0 + (seed % 9973) / 9973.0)
        st["cos"] = torch.zeros((case["n_pos"], half), device="cuda")
        st["sin"] = torch.zeros((case["n_pos"], half), device="cuda")
        return st
    if kind == "rope":
        R, nq, nkv, hd, page = case["R"], case["nq"], case["nkv"], case["hd"], case["page"]
        tx, ty = TYPES[case["x"]], TYPES[case["y"]]
        n_pos, half = 4096, case["rot"] // 2
        qkv = (torch.randn((R, (nq + 2 * nkv) * hd), generator=gen, device="cuda") *
               torch.exp(0.5 * torch.randn((R, 1), generator=gen, device="cuda"))).to(tx)
        st["q"] = qkv[:, : nq * hd].unflatten(1, (nq, hd))
        st["k"] = qkv[:, nq * hd: (nq + nkv) * hd].unflatten(1, (nkv, hd))
        st["v"] = qkv[:, (nq + nkv) * hd:].unflatten(1, (nkv, hd))
        ang = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * \
            THETA ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)[None, :]
        st["cos"], st["sin"] = torch.cos(ang).float(), torch.sin(ang).float()
        pos = torch.randint(0, n_pos, (R,), generator=gen, device="cuda", dtype=torch.int32)
        n_pages = (R + page - 1) // page + 2
        # runs of positions fill pages that lie anywhere in the pool
        pages = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        at = torch.arange(R, device="cuda", dtype=torch.int32)
        slot = pages[(at // page).long()] * page + at % page
        if case["pad"]:
            none = torch.rand(R, generator=gen, device="cuda") < case["pad"]
            pos[none], slot[none] = -1, -1
        st["pos"], st["slot"] = pos, slot
        st["q_out"] = torch.zeros((R, nq, hd), dtype=ty, device="cuda")
        st["k_pages"] = torch.zeros((n_pages, nkv, page, hd), dtype=ty, device="cuda")
        st["v_pages"] = torch.zeros((n_pages, nkv, page, hd), dtype=ty, device="cuda")
        return st
    if kind == "verify":
        V, t, counts = case["vocab"], TYPES[case["t"]], _drafts(case)
        D, B = sum(counts), case["B"]
        st["draft_start"] = _starts(counts)
        logits = _probabilities(gen, D + B, V)
        st["p"] = _filtered(logits, case["top"], t)
        # the draft approximates the target's rows; the last row of every sequence has no draft
        seq = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(counts, device="cuda"))
        q = _filtered(_probabilities(gen, D, V, near=logits[torch.arange(D, device="cuda") + seq]), case["top"], t)
        if D:
            st["drafted"] = torch.multinomial(q.float(), 1, generator=gen)[:, 0].to(torch.int32)
        else:
            st["drafted"] = torch.zeros(0, dtype=torch.int32, device="cuda")
        st["q"] = q if case["q"] else None  # without: drafts looked up in the text, each the only one its row could give
        st["u_accept"] = torch.rand(D, generator=gen, device="cuda")
        st["u_next"] = torch.rand(B, generator=gen, device="cuda")
        st["accepted"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        st["token"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        if own:
            import paper_2504_00030_amd as pk
            st["workspace"] = torch.empty(pk.k_verify_workspace(B, V), dtype=torch.uint8, device="cuda")
        return st
    nq, nkv, hd, page, t = case["nq"], case["nkv"], case["hd"], case["page"], TYPES[case["t"]]
    rows, lens = _lengths(case)
    B, R, prefix = case["B"], sum(rows), case["prefix"]
    most = max(lens)
    n_prefix, n_own = (prefix + page - 1) // page, (most + page - 1) // page
    n_pages = n_prefix + B * n_own + 1
    st["q"] = (1.5 * torch.randn((R, nq, hd), generator=gen, device="cuda")).to(t)
    chan = torch.exp(0.3 * torch.randn((nkv, 1, hd), generator=gen, device="cuda"))
    st["k_pages"] = (torch.randn((n_pages, nkv, page, hd), generator=gen, device="cuda") * chan).to(t)
    st["v_pages"] = torch.randn((n_pages, nkv, page, hd), generator=gen, device="cuda").to(t)
    perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    st["prefix_table"] = perm[:n_prefix].contiguous()
    st["table"] = perm[n_prefix: n_prefix + B * n_own].reshape(B, n_own).contiguous()
    st["row_start"] = _starts(rows)
    st["own_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st["out"] = torch.zeros((R, nq, hd), dtype=t, device="cuda")
    if own:
        import paper_2504_00030_amd as pk
        n = pk.k_attn_shared_workspace(R, B, nq, nkv, hd, t, prefix, n_own * page)
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st


def _frequencies(case, theta):
    """Plain form: radians a position, in 64 bits, and the factor of both tables."""
    rot, a = case["rot"], SCALED[case["scaling"]]
    half = rot // 2
    at = torch.arange(half, device="cuda", dtype=torch.float64)
    f = theta ** (-at / half)
    if case["scaling"] == "linear":
        return f / a["factor"], 1.0
    if case["scaling"] == "base":
        return (theta * a["factor"] ** (rot / max(rot - 2, 1))) ** (-at / half), 1.0
    if case["scaling"] == "bands":
        keep = ((a["context"] * f / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / a["factor"]), 1.0
    if case["scaling"] == "ramp":
        first, last = (half * math.log(a["context"] / (2 * math.pi * n)) / math.log(theta) for n in (a["high"], a["low"]))
        first, last = max(math.floor(first), 0), min(math.ceil(last), rot - 1)
        gone = ((at - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
        return f * (1.0 - gone + gone / a["factor"]), 0.1 * math.log(a["factor"]) + 1.0
    return f, 1.0


def _rotated(h, cos, sin, rot, inter):
    if inter:
        a, b = h[..., 0:rot:2], h[..., 1:rot:2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = h[..., : rot // 2], h[..., rot // 2: rot]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([r, h[..., rot:]], dim=-1)


def _attention(st):
    """Plain form: scores of all rows against the prefix in one product a head, against their own positions in a padded one."""
    case, q = st["case"], st["q"].float()
    R, nq, hd = q.shape
    nkv, page, B, prefix = case["nkv"], case["page"], case["B"], case["prefix"]
    g = nq // nkv
    q = q.reshape(R, nkv, g, hd).transpose(0, 1)  # [kv head][row][query head of it]
    rows = case["rows"]
    start = st["row_start"].long()
    count = start[1:] - start[:-1]
    idx = start[:-1, None] + torch.arange(rows, device="cuda")[None, :]
    there = torch.arange(rows, device="cuda")[None, :] < count[:, None]  # [B][rows]
    back = (torch.arange(R, device="cuda")[:, None] >= start[None, 1:]).sum(dim=1)  # sequence of a row
    back = back * rows + torch.arange(R, device="cuda") - start[back]
    qp = q[:, idx.clamp(max=R - 1)]  # [kv head][B][rows][g][hd]
    k = st["k_pages"][st["table"].long()].float().permute(2, 0, 1, 3, 4).reshape(nkv, B, -1, hd)
    v = st["v_pages"][st["table"].long()].float().permute(2, 0, 1, 3, 4).reshape(nkv, B, -1, hd)
    L = k.shape[2]
    s = (qp.reshape(nkv, B, rows * g, hd) @ k.transpose(2, 3).contiguous()).reshape(nkv, B, rows, g, L) * hd ** -0.5
    last = st["own_len"].long()[:, None] - count[:, None] + torch.arange(rows, device="cuda")[None, :]
    seen = (torch.arange(L, device="cuda")[None, None, :] <= last[:, :, None]) & there[:, :, None]
    s = torch.where(seen[None, :, :, None, :], s, torch.full_like(s, -math.inf))
    own_s = s.reshape(nkv, B * rows, g, L)[:, back]  # [kv head][row][g][L]
    m = own_s.amax(dim=-1, keepdim=True)
    if prefix:
        kp = st["k_pages"][st["prefix_table"].long()].float().permute(1, 0, 2, 3).reshape(nkv, -1, hd)[:, :prefix]
        vp = st["v_pages"][st["prefix_table"].long()].float().permute(1, 0, 2, 3).reshape(nkv, -1, hd)[:, :prefix]
        sp = (q.reshape(nkv, R * g, hd) @ kp.transpose(1, 2).contiguous()).reshape(nkv, R, g, prefix) * hd ** -0.5
        m = torch.maximum(m, sp.amax(dim=-1, keepdim=True))
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(own_s - m)
    total = e.sum(dim=-1, keepdim=True)
    ep = torch.zeros((nkv, B * rows, g, L), device="cuda")
    ep[:, back] = e
    o = (ep.reshape(nkv, B, rows * g, L) @ v).reshape(nkv, B * rows, g, hd)[:, back]
    if prefix:
        e = torch.exp(sp - m)
        total = total + e.sum(dim=-1, keepdim=True)
        o = o + (e.reshape(nkv, R * g, prefix) @ vp).reshape(nkv, R, g, hd)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.transpose(0, 1).reshape(R, nq, hd).to(st["out"].dtype)


def _verified(st):
    p, q, ds = st["p"], st["q"], st["draft_start"].long()
    B, D, V = ds.shape[0] - 1, st["drafted"].shape[0], p.shape[1]
    seqs = torch.arange(B, device="cuda")
    k = ds[1:] - ds[:-1]
    n = torch.arange(D, device="cuda")
    seq = (n[:, None] >= ds[None, 1:]).sum(dim=1)
    x = st["drafted"].long()
    px = p[n + seq, x].double()
    qx = q[n, x].double() if q is not None else torch.ones(D, dtype=torch.float64, device="cuda")
    kept = st["u_accept"].double() * qx < px
    # accepted: drafts in front of the first one that was not kept
    first = torch.where(kept, k[seq], n - ds[seq])
    A = k.scatter_reduce(0, seq, first, "amin", include_self=True)
    w = p[ds[:-1] + seqs + A].double()
    if D:
        refused = (ds[:-1] + A).clamp(max=D - 1)
        if q is not None:
            rest = (w - q[refused].double()).clamp_min(0.0)
        else:
            rest = w.scatter(1, x[refused][:, None], 0.0)
        use = (A < k)[:, None] & (rest.sum(dim=1, keepdim=True) > 0)
        w = torch.where(use, rest, w)
    c = torch.cumsum(w, dim=1)
    above = c > st["u_next"].double()[:, None] * c[:, -1:]
    places = torch.arange(V, device="cuda")
    behind = torch.where(w > 0, places, torch.zeros_like(places)).amax(dim=1)
    y = torch.where(above.any(dim=1), above.to(torch.int32).argmax(dim=1), behind)
    return {"accepted": A.to(torch.int32), "token": y.to(torch.int32)}


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        import paper_2504_00030_amd as pk
        stream = torch.cuda.current_stream().cuda_stream
        if kind == "tables":
            pk.k_rope_tables(state["cos"], state["sin"], theta=state["theta"], scaling=case["scaling"], stream=stream, **SCALED[case["scaling"]])
            return {"cos": state["cos"], "sin": state["sin"]}
        if kind == "rope":
            pk.k_rope_cache(state["q"], state["k"], state["v"], state["cos"], state["sin"], state["pos"], state["slot"], state["q_out"],
                            state["k_pages"], state["v_pages"], interleaved=case["inter"], stream=stream)
            return {"q": state["q_out"], "k": state["k_pages"], "v": state["v_pages"]}
        if kind == "attn":
            pk.k_attn_shared(state["q"], state["k_pages"], state["v_pages"], state["row_start"], state["table"], state["own_len"],
                             state["out"], state["workspace"], prefix_table=state["prefix_table"], prefix_len=case["prefix"], stream=stream)
            return {"o": state["out"]}
        pk.k_verify(state["p"], state["q"], state["draft_start"], state["drafted"], state["u_accept"], state["u_next"],
                    state["accepted"], state["token"], state["workspace"], stream=stream)
        return {"accepted": state["accepted"], "token": state["token"]}
    if kind == "tables":
        f, size = _frequencies(case, state["theta"])
        ang = torch.arange(case["n_pos"], device="cuda", dtype=torch.float64)[:, None] * f[None, :]
        return {"cos": (torch.cos(ang) * size).float(), "sin": (torch.sin(ang) * size).float()}
    if kind == "rope":
        pos, slot, page = state["pos"], state["slot"], case["page"]
        kp, vp, n_pos = state["k_pages"], state["v_pages"], state["cos"].shape[0]
        there = (pos >= 0) & (pos < n_pos)
        at = pos.clamp(0, n_pos - 1).long()
        c, s = state["cos"][at][:, None, :], state["sin"][at][:, None, :]
        q = _rotated(state["q"].float(), c, s, case["rot"], case["inter"]).to(kp.dtype)
        k = _rotated(state["k"].float(), c, s, case["rot"], case["inter"]).to(kp.dtype)
        q = torch.where(there[:, None, None], q, state["q_out"])
        kept = there & (slot >= 0) & (slot < kp.shape[0] * page)
        to = slot[kept].long()
        kp[to // page, :, to % page] = k[kept]
        vp[to // page, :, to % page] = state["v"][kept].to(vp.dtype)
        return {"q": q, "k": kp, "v": vp}
    if kind == "attn":
        return {"o": _attention(state)}
    return _verified(state)


def work(case):
    kind = case["kind"]
    if kind == "tables":
        n = case["n_pos"] * case["rot"] // 2
        return {"bytes": 8.0 * n, "flops": 4.0 * n}
    if kind == "rope":
        rows = case["R"] * (1.0 - case["pad"])
        n = rows * (case["nq"] + 2 * case["nkv"]) * case["hd"]
        turned = rows * (case["nq"] + case["nkv"]) * case["rot"]
        return {"bytes": n * (SIZE[case["x"]] + SIZE[case["y"]]) + min(rows, 4096.0) * case["rot"] * 4.0 + 8.0 * case["R"],
                "flops": 3.0 * turned}
    if kind == "verify":
        # the two probabilities of every draft, and the rows of one draw a sequence: both models', or the target's
        counts = _drafts(case)
        size = SIZE[case["t"]]
        rows = sum(2.0 if k and case["q"] else 1.0 for k in counts)
        return {"bytes": rows * case["vocab"] * size + sum(counts) * (8.0 + 2.0 * size) + 20.0 * case["B"], "flops": 3.0 * case["B"] * case["vocab"]}
    rows, lens = _lengths(case)
    size, nq, nkv, hd = SIZE[case["t"]], case["nq"], case["nkv"], case["hd"]
    positions = case["prefix"] + sum(lens)
    pairs = sum(r * (case["prefix"] + n) - r * (r - 1) / 2.0 for r, n in zip(rows, lens))
    return {"bytes": (2.0 * positions * nkv + 2.0 * sum(rows) * nq) * hd * size, "flops": 4.0 * pairs * nq * hd}


def _exact_frequencies(case, theta):
    """Radians a position by the definition, one frequency after the other."""
    rot, a, name = case["rot"], SCALED[case["scaling"]], case["scaling"]
    out = []
    for j in range(rot // 2):
        f = math.exp(-2.0 * j / rot * math.log(theta))
        if name == "linear":
            f /= a["factor"]
        elif name == "base":
            f = math.exp(-2.0 * j / rot * (math.log(theta) + rot / max(rot - 2, 1) * math.log(a["factor"])))
        elif name == "bands":
            turns = a["context"] * f / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - a["low"]) / (a["high"] - a["low"])))
            f = keep * f + (1.0 - keep) * f / a["factor"]
        elif name == "ramp":
            edge = [rot * math.log(a["context"] / (2.0 * math.pi * n)) / (2.0 * math.log(theta)) for n in (a["high"], a["low"])]
            lo, hi = max(0, math.floor(edge[0])), min(rot - 1, math.ceil(edge[1]))
            gone = min(1.0, max(0.0, (j - lo) / max(0.001, hi - lo)))
            f = (1.0 - gone) * f + gone * f / a["factor"]
        out.append(f)
    return out, (1.0 + 0.1 * math.log(a["factor"]) if name == "ramp" else 1.0)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "tables":
        f, size = _exact_frequencies(case, st["theta"])
        pos = torch.arange(case["n_pos"], device="cuda", dtype=torch.float64)
        turn = torch.polar(torch.full((case["n_pos"], len(f)), size, dtype=torch.float64, device="cuda"),
                           torch.outer(pos, torch.tensor(f, dtype=torch.float64, device="cuda")))
        return {"cos": turn.real.contiguous(), "sin": turn.imag.contiguous()}
    if kind == "rope":
        rot, page = case["rot"], case["page"]
        res = {"q": st["q_out"].double(), "k": st["k_pages"].double(), "v": st["v_pages"].double()}
        for rows in torch.nonzero(st["pos"] >= 0).flatten().split(4096):
            at = st["pos"][rows].long()
            turn = torch.complex(st["cos"][at].double(), st["sin"][at].double()).unsqueeze(1)
            slot = st["slot"][rows].long()
            for name in ("q", "k"):
                h = st[name][rows].double()
                first, second = (slice(0, rot, 2), slice(1, rot, 2)) if case["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
                z = torch.complex(h[..., first], h[..., second]) * turn
                h[..., first], h[..., second] = z.real, z.imag
                if name == "q":
                    res["q"][rows] = h
                else:
                    res["k"].transpose(1, 2)[slot // page, slot % page] = h
            res["v"].transpose(1, 2)[slot // page, slot % page] = st["v"][rows].double()
        return res
    if kind == "verify":
        start = st["draft_start"].tolist()
        drafted, ua, un = st["drafted"].tolist(), st["u_accept"].tolist(), st["u_next"].tolist()
        accepted, tokens = [], []
        for b in range(case["B"]):
            first, k, A = start[b], start[b + 1] - start[b], 0
            p = st["p"][first + b: first + b + k + 1].double().cpu()
            while A < k:
                x = drafted[first + A]
                give = float(st["q"][first + A, x]) if st["q"] is not None else 1.0
                if not ua[first + A] * give < float(p[A, x]):
                    break
                A += 1
            w = p[A]
            if A < k:
                if st["q"] is not None:
                    rest = torch.clamp(w - st["q"][first + A].double().cpu(), min=0.0)
                else:
                    rest = w.clone()
                    rest[drafted[first + A]] = 0.0
                w = rest if bool((rest > 0).any()) else w
            c = torch.cumsum(w, dim=0)
            y = int(torch.searchsorted(c, un[b] * float(c[-1]), right=True))
            accepted.append(A)
            tokens.append(y if y < case["vocab"] else int(torch.nonzero(w > 0).max()))
        return {"accepted": torch.tensor(accepted, dtype=torch.int32, device="cuda"), "token": torch.tensor(tokens, dtype=torch.int32, device="cuda")}
    rows, lens = _lengths(case)
    nq, nkv, hd, prefix = case["nq"], case["nkv"], case["hd"], case["prefix"]
    g = nq // nkv
    out = torch.zeros((sum(rows), nq, hd), dtype=torch.float64, device="cuda")
    r0 = 0
    for b, (n, L) in enumerate(zip(rows, lens)):
        own_at = torch.arange(L, device="cuda")
        page_of = torch.cat([st["prefix_table"].long().repeat_interleave(case["page"])[:prefix], st["table"][b].long()[own_at // case["page"]]])
        place = torch.cat([torch.arange(prefix, device="cuda") % case["page"], own_at % case["page"]])
        hide = torch.zeros((n, prefix + L), dtype=torch.bool, device="cuda")
        hide[:, prefix:] = own_at[None, :] > (L - n + torch.arange(n, device="cuda"))[:, None]
        for h in range(nkv):
            k = st["k_pages"][page_of, h, place].double()
            v = st["v_pages"][page_of, h, place].double()
            for i in range(g):
                s = st["q"][r0: r0 + n, h * g + i].double() @ k.t() / math.sqrt(hd)
                out[r0: r0 + n, h * g + i] = torch.softmax(s.masked_fill(hide, -math.inf), dim=1) @ v
        r0 += n
    return {"o": out}
