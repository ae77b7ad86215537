"""The operators around the Spense linear layers that are timed: norms before and after a block,
low-rank adapters beside a projection, and products grouped by expert.

listed() names the cases, draw() gives more of the same ranges.  prepare() makes what a program
holds before the call, run() is one pass: the plain form in elementary torch operations, or, with
``own`` set, the package's public entry points.  exact() is the definition in 64 bits, work() what
a pass cannot do without.

Weights are N(0, 0.02), pruned 2:4 by magnitude, with per-row absmax / 448 scales; activations are
N(0, 1) with a few large channels.
"""
from __future__ import annotations

import torch

own = False

FP8_MAX = 448.0
EPS = 1e-6


def listed():
    return [
        # the norm in front of the first block for one decoding sequence: the smallest call
        {"name": "norm_m1", "op": "norm", "M": 1, "K": 5120, "type": "bf16", "post": False, "gate": "none",
         "normed": False},
        # between attention and MLP of a full decode batch: post-norm, channel gate, residual, pre-norm, codes
        {"name": "norm_m64", "op": "norm", "M": 64, "K": 5120, "type": "bf16", "post": True, "gate": "channel",
         "normed": False},
        # an odd hidden size with an fp32 stream on a ragged chunk of a prompt, a gate per token
        {"name": "norm_m517_odd", "op": "norm", "M": 517, "K": 4099, "type": "f32", "post": True, "gate": "token",
         "normed": True},
        # a long prompt chunk, with the bf16 output for the adapters beside the codes
        {"name": "norm_m8192", "op": "norm", "M": 8192, "K": 5120, "type": "bf16", "post": True, "gate": "channel",
         "normed": True},
        # two sequences with small adapters on a k / v projection
        {"name": "adapters_m2", "op": "adapters", "M": 2, "K": 5120, "N": 1024, "R": 8, "count": 4, "x": "fp8",
         "base": "f32", "run_len": 1},
        # a decode batch of many requests on a gate / up projection
        {"name": "adapters_m64", "op": "adapters", "M": 64, "K": 5120, "N": 25600, "R": 16, "count": 32, "x": "fp8",
         "base": "f32", "run_len": 1},
        # prompts of several requests on a q projection, from the norm's bf16 output
        {"name": "adapters_m2048", "op": "adapters", "M": 2048, "K": 5120, "N": 8192, "R": 64, "count": 16, "x": "bf16",
         "base": "f32", "run_len": 150},
        # gate and up of a decode batch: every expert gets a few tokens
        {"name": "experts_t32", "op": "experts", "T": 32, "top": 8, "E": 64, "N": 1536, "K": 5120, "split": "output",
         "dense_frac": 0.25, "pair": True},
        # the input-split down projection of a ragged batch
        {"name": "experts_down_t150", "op": "experts", "T": 150, "top": 6, "E": 40, "N": 5120, "K": 1408,
         "split": "input", "dense_frac": 0.25, "pair": False},
        # gate and up of a prompt chunk
        {"name": "experts_t4096", "op": "experts", "T": 4096, "top": 4, "E": 16, "N": 2560, "K": 5120,
         "split": "output", "dense_frac": 0.25, "pair": True},
        # the whole MLP of experts for one decoding sequence
        {"name": "mlp_t1", "op": "mlp", "T": 1, "top": 8, "E": 32, "hidden": 5120, "inter": 1536, "dense_frac": 0.25},
        # and for a prompt chunk
        {"name": "mlp_t2048", "op": "mlp", "T": 2048, "top": 4, "E": 32, "hidden": 5120, "inter": 1536,
         "dense_frac": 0.25},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["norm", "norm", "adapters", "adapters", "experts", "experts", "experts", "mlp"])
    if op == "norm":
        K = _log(rng, 128, 12288)
        K = K if rng.random() < 0.3 else max(128, K // 64 * 64)
        M = _log(rng, 1, min(8192, 8192 * 5120 // K))
        post = rng.random() < 0.7
        return {"op": op, "M": M, "K": K, "type": rng.choice(["bf16", "bf16", "f32"]), "post": post,
                "gate": rng.choice(["none", "channel", "token"]) if post else "none", "normed": rng.random() < 0.5}
    if op == "adapters":
        M, N, K = _log(rng, 1, 2048), _log(rng, 256, 25600), 32 * _log(rng, 16, 800)
        if M * N > 2048 * 8192:
            M = max(1, 2048 * 8192 // N)
        R = rng.choice([8, 16, 16, 32, 64])
        if M > 256:
            K = min(K, 5120)
        return {"op": op, "M": M, "K": K, "N": N, "R": R, "count": _log(rng, 1, 32),
                "x": rng.choice(["fp8", "bf16"]), "base": rng.choice(["f32", "f32", "bf16"]),
                "run_len": 1 if M <= 128 else rng.choice([1, 40, 150, 600])}
    frac = rng.choice([0.0, 0.25, 0.25, 0.5, 1.0])
    E = _log(rng, 4, 64)
    top = min(E, rng.choice([1, 2, 4, 6, 8]))
    T = min(_log(rng, 1, 4096), 16384 // top)
    if op == "mlp":
        hidden, inter = 256 * rng.randint(4, 20), 128 * rng.randint(4, 14)
        return {"op": op, "T": min(T, 8192 // top), "top": top, "E": min(E, 32), "hidden": hidden, "inter": inter,
                "dense_frac": frac}
    split = rng.choice(["output", "input"])
    N = _log(rng, 256, 2560) if split == "output" else _log(rng, 1024, 5120)
    K = 32 * _log(rng, 32, 160 if split == "output" else 80)
    return {"op": op, "T": T, "top": top, "E": E if N * K * E <= 64 * 1536 * 5120 else max(top, E // 4), "N": N, "K": K,
            "split": split, "dense_frac": frac, "pair": split == "output" and rng.random() < 0.6}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _act(g, M, K):
    """Activations: N(0, 1) with log-normal channel scales, about one channel in 256 ten times larger."""
    ch = torch.exp(0.3 * _randn(g, K))
    big = torch.rand(K, generator=g, device="cuda") < 1 / 256
    return _randn(g, M, K) * torch.where(big, 10 * ch, ch)


def _codes(a):
    """Per-row absmax / 448 scales and e4m3fn values (as float8) of an fp32 tensor."""
    s = a.abs().amax(-1)
    s = s / torch.full_like(s, FP8_MAX)
    s = torch.where(s == 0, torch.ones_like(s), s)
    return (a / s[..., None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn), s


def _prune24(w, split, db):
    """w (E x N x K) with the two smaller magnitudes of each group of four of the 2:4 region zeroed."""
    reg = w[:, :db] if split == "output" else w[:, :, :db]
    if reg.numel():
        a = reg.reshape(reg.shape[0], reg.shape[1], -1, 4)
        m, i = a.abs(), torch.arange(4, device=a.device)
        ahead = m[..., None, :] > m[..., :, None]
        ahead |= (m[..., None, :] == m[..., :, None]) & (i[None, :] < i[:, None])  # ties: the lower index
        keep = ahead.sum(-1, dtype=torch.uint8) < 2
        reg.copy_(torch.where(keep, a, torch.zeros_like(a)).reshape(reg.shape))
    return w


def _dense_begin(extent, frac, granule):
    """First index of the trailing dense region."""
    return min(extent, int(round((extent - round(frac * extent)) / granule)) * granule)


def _expert_weights(g, E, N, K, split, frac):
    """{codes: E x N x K float8 with zeros where pruned, scale: E x N, packed (for the kernels)}."""
    db = _dense_begin(N if split == "output" else K, frac, 16 if split == "output" else 32)
    codes = torch.empty((E, N, K), dtype=torch.float8_e4m3fn, device="cuda")
    scale = torch.empty((E, N), device="cuda")
    for e in range(E):
        q, s = _codes(_prune24(_randn(g, 1, N, K).mul_(0.02), split, db))
        codes[e], scale[e] = q[0], s[0]
    out = {"codes": codes, "scale": scale}
    if own:
        import paper_2606_10445_amd as S

        axis = S.SPENSE_SPLIT_OUTPUT if split == "output" else S.SPENSE_SPLIT_INPUT
        out["packed"] = S.stack_experts([S.tile(S.compress(codes[e].view(torch.uint8), None, axis, db))
                                         for e in range(E)])
    return out


def _routing(g, T, top, E):
    """Expert of each token's choices (T x top int32, distinct) and their weights (T x top, sum 1); experts
    differ in how often they are chosen."""
    logits = _randn(g, T, E) + 0.5 * _randn(g, E)
    v, i = torch.topk(logits, top, dim=1)
    return i.to(torch.int32), torch.softmax(v, 1)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    op = case["op"]
    if op == "norm":
        M, K = case["M"], case["K"]
        dt = torch.bfloat16 if case["type"] == "bf16" else torch.float32
        s["x"] = (4 * _act(g, M, K)).to(dt)
        s["weight"] = (1 + 0.1 * _randn(g, K)).to(dt)
        s["y"] = _act(g, M, K).to(dt) if case["post"] else None
        s["post_weight"] = (1 + 0.1 * _randn(g, K)).to(dt) if case["post"] else None
        s["gate"] = {"none": None, "channel": _randn(g, K).mul_(0.5).to(dt),
                     "token": _randn(g, M, K).mul_(0.5).to(dt)}[case["gate"]]
        s["alpha"] = 0.875
    elif op == "adapters":
        M, K, N, R, count = (case[k] for k in ("M", "K", "N", "R", "count"))
        x = _act(g, M, K)
        s["X"], s["x_scale"] = _codes(x) if case["x"] == "fp8" else (x.bfloat16(), None)
        # requests of about run_len consecutive tokens, one in eight without an adapter
        runs = -(-M // case["run_len"])
        idx = torch.randint(0, count, (runs,), generator=g, device="cuda")
        idx = torch.where(torch.rand(runs, generator=g, device="cuda") < 0.125, torch.full_like(idx, -1), idx)
        s["idx"] = idx.repeat_interleave(case["run_len"])[:M].to(torch.int32)
        s["A"] = _randn(g, count, R, K).mul_(K ** -0.5).bfloat16()
        s["B"] = _randn(g, count, N, R).mul_(0.5 * R ** -0.5).bfloat16()
        s["scale"] = 0.5 + torch.rand(count, generator=g, device="cuda")
        s["base"] = _randn(g, M, N).to(torch.float32 if case["base"] == "f32" else torch.bfloat16)
        if own:
            import paper_2606_10445_amd as S

            s["pool"] = S.AdapterPool(s["A"], s["B"], s["scale"])
    else:
        T, top, E = case["T"], case["top"], case["E"]
        K = case["K"] if op == "experts" else case["hidden"]
        s["idx"], s["weights"] = _routing(g, T, top, E)
        # rows of the fullest expert: the plain form pads every expert to it
        s["cap"] = int(torch.bincount(s["idx"].flatten().long(), minlength=E).max())
        s["X"], s["x_scale"] = _codes(_act(g, T, K))
        if op == "experts":
            s["w"] = [_expert_weights(g, E, case["N"], K, case["split"], case["dense_frac"])
                      for _ in range(2 if case["pair"] else 1)]
        else:
            I = case["inter"]
            s["w"] = [_expert_weights(g, E, I, K, "output", case["dense_frac"]),
                      _expert_weights(g, E, I, K, "output", case["dense_frac"]),
                      _expert_weights(g, E, K, I, "input", case["dense_frac"])]
    return s


# ------------------------------------------------------------------ the plain forms
def _rms(v, w):
    n = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return n * w.float() if w is not None else n


def _dequant(q, scale):
    """The values that codes and scales stand for, in bf16."""
    return (q.float() * scale[:, None]).bfloat16()


def _plain_norm(s):
    r = s["x"].float()
    if s["y"] is not None:
        t = _rms(s["y"].float(), s["post_weight"])
        r = s["alpha"] * r + (t if s["gate"] is None else s["gate"].float() * t)
    n = _rms(r, s["weight"])
    q, scale = _codes(n)
    return {"residual": r.to(s["x"].dtype) if s["y"] is not None else None,
            "normed": n.to(s["x"].dtype) if s["case"]["normed"] else None, "values": _dequant(q, scale), "scales": scale}


def _plain_adapters(s):
    """Every adapter's low-rank activations of every token, those of other adapters masked out."""
    count, R, K = s["A"].shape
    M = s["X"].shape[0]
    V = s["X"].float() @ s["A"].float().reshape(count * R, K).t()
    if s["x_scale"] is not None:
        V = V * s["x_scale"][:, None]
    mine = s["idx"][:, None] == torch.arange(count, device=V.device)[None, :]
    V = V.reshape(M, count, R) * (mine * s["scale"][None, :])[:, :, None]
    B = s["B"].float().permute(0, 2, 1).reshape(count * R, -1)
    return (s["base"].float() + V.reshape(M, count * R) @ B).bfloat16()


def _plain_group(idx, E):
    """(order, expert and slot inside its expert of each position) of the rows sorted by expert, stable."""
    flat = idx.reshape(-1).long()
    e, order = torch.sort(flat, stable=True)
    first = torch.cumsum(torch.bincount(flat, minlength=E), 0) - torch.bincount(flat, minlength=E)
    return order, e, torch.arange(flat.numel(), device=flat.device) - first[e]


def _plain_product(x, x_scale, e, slot, cap, w):
    """x[p] W[e[p]]^T in fp32, every expert padded to cap rows."""
    E, N, K = w["codes"].shape
    pad = torch.zeros((E, cap, K), device=x.device)
    pad[e, slot] = x.float()
    y = torch.bmm(pad, w["codes"].float().transpose(1, 2).contiguous())[e, slot]
    return y * w["scale"][e] * x_scale[:, None]


def _plain_experts(s):
    E = s["w"][0]["codes"].shape[0]
    order, e, slot = _plain_group(s["idx"], E)
    rows = order // s["case"]["top"]
    x, xs = s["X"][rows], s["x_scale"][rows]
    return [order.to(torch.int32)] + [_plain_product(x, xs, e, slot, s["cap"], w).bfloat16() for w in s["w"]]


def _plain_mlp(s):
    E = s["w"][0]["codes"].shape[0]
    T, top = s["idx"].shape
    order, e, slot = _plain_group(s["idx"], E)
    rows = order // top
    x, xs = s["X"][rows], s["x_scale"][rows]
    gate, up, down = s["w"]
    g = _plain_product(x, xs, e, slot, s["cap"], gate)
    u = _plain_product(x, xs, e, slot, s["cap"], up)
    hq, hs = _codes(u * g / (1 + torch.exp(-g)))
    d = _plain_product(hq, hs, e, slot, s["cap"], down) * s["weights"].reshape(-1)[order][:, None]
    y = torch.empty_like(d)
    y[order] = d
    return y.reshape(T, top, -1).sum(1).bfloat16()


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "adapters": _plain_adapters, "experts": _plain_experts, "mlp": _plain_mlp}[op](s)
    import paper_2606_10445_amd as S

    if op == "norm":
        o = S.block_norm(s["x"], s["y"], post_weight=s["post_weight"], gate=s["gate"], residual_scale=s["alpha"],
                         weight=s["weight"], eps=EPS, normed=s["case"]["normed"], quantize=True)
        return {"residual": o.residual if s["y"] is not None else None, "normed": o.normed,
                "values": _dequant(o.codes.view(torch.float8_e4m3fn), o.scales), "scales": o.scales}
    if op == "adapters":
        groups = S.group_rows(s["idx"], s["pool"].count)
        return S.add_adapters(s["base"], s["X"], s["pool"], groups, x_scale=s["x_scale"])
    if op == "experts":
        groups = S.group_rows(s["idx"].view(-1), s["case"]["E"])
        ys = S.gemm_experts(s["X"], [w["packed"] for w in s["w"]], groups, [w["scale"] for w in s["w"]], s["x_scale"],
                            top=s["case"]["top"])
        return [groups.order] + ys
    gate, up, down = s["w"]
    return S.mlp_experts(s["X"], s["x_scale"], s["idx"], s["weights"], gate["packed"], up["packed"], down["packed"],
                         gate["scale"], up["scale"], down["scale"])


# ------------------------------------------------------------------ in 64 bits
def _exact_codes(a):
    """fp32 scales and the e4m3fn values of a float64 tensor's rows, as float64."""
    s = (a.abs().amax(1) / FP8_MAX).float().double()
    s = torch.where(s == 0, torch.ones_like(s), s)
    v = (a / s[:, None]).clamp(-FP8_MAX, FP8_MAX)
    # three fraction bits, and steps of 2^-9 below 2^-6; round() takes ties to even
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step, s


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        def norm(v, w):
            return v / torch.sqrt(v.pow(2).sum(1, keepdim=True) / v.shape[1] + EPS) * w.double()

        r = s["x"].double()
        if case["post"]:
            t = norm(s["y"].double(), s["post_weight"])
            if case["gate"] != "none":
                t = t * s["gate"].double()
            r = r * s["alpha"] + t
        n = norm(r, s["weight"])
        q, scale = _exact_codes(n)
        return {"residual": r if case["post"] else None, "normed": n if case["normed"] else None,
                "values": q * scale[:, None], "scales": scale}
    if op == "adapters":
        x = s["X"].double() if s["x_scale"] is None else s["X"].double() * s["x_scale"].double()[:, None]
        y = s["base"].double()
        idx = s["idx"].tolist()
        for a in range(case["count"]):
            m = [i for i, k in enumerate(idx) if k == a]
            if m:
                v = x[m] @ s["A"][a].double().t()
                y[m] += s["scale"][a].double() * (v @ s["B"][a].double().t())
        return y
    E, top = case["E"], case["top"]
    flat = s["idx"].reshape(-1).tolist()
    where = [[i for i, e in enumerate(flat) if e == k] for k in range(E)]
    x = s["X"].double() * s["x_scale"].double()[:, None]

    def weight(w, e):
        return w["codes"][e].double() * w["scale"][e].double()[:, None]

    if op == "experts":
        order = [i for rows in where for i in rows]
        outs = [[x[[i // top for i in rows]] @ weight(w, e).t() for e, rows in enumerate(where) if rows] for w in s["w"]]
        return [torch.tensor(order, dtype=torch.int32, device="cuda")] + [torch.cat(o) for o in outs]
    gate, up, down = s["w"]
    y = torch.zeros((case["T"], case["hidden"]), dtype=torch.float64, device="cuda")
    for e, rows in enumerate(where):
        if not rows:
            continue
        tok = [i // top for i in rows]
        g, u = x[tok] @ weight(gate, e).t(), x[tok] @ weight(up, e).t()
        hq, hs = _exact_codes(u * g / (1 + torch.exp(-g)))
        d = (hq * hs[:, None]) @ weight(down, e).t()
        y[tok] += s["weights"].reshape(-1)[rows].double()[:, None] * d  # a token's experts are distinct
    return y


# ------------------------------------------------------------------ what a pass cannot do without
def _entry_bytes(N, K, split, frac):
    """Stored bytes and multiplied entries of one expert's weight (2:4: values and 4 bits per group of four)."""
    extent = N if split == "output" else K
    db = _dense_begin(extent, frac, 16 if split == "output" else 32)
    sparse = db * (K if split == "output" else N)
    return N * K - sparse + 0.625 * sparse, N * K - sparse / 2


def work(case):
    op = case["op"]
    if op == "norm":
        M, K = case["M"], case["K"]
        es = 2 if case["type"] == "bf16" else 4
        per = es + 1 + (es if case["normed"] else 0)  # x, codes, normed
        vec = es * K
        if case["post"]:
            per += 2 * es + (es if case["gate"] == "token" else 0)  # y, residual, gate
            vec += es * K + (es * K if case["gate"] == "channel" else 0)
        return {"bytes": M * K * per + vec + 4 * M, "flops": 12 * M * K}
    if op == "adapters":
        M, K, N, R = (case[k] for k in ("M", "K", "N", "R"))
        used = min(case["count"], -(-M // case["run_len"]))
        x = M * K * (1 if case["x"] == "fp8" else 2)
        y = M * N * ((4 if case["base"] == "f32" else 2) + 2)
        return {"bytes": x + y + used * 2 * R * (K + N) + 8 * M, "flops": 2 * M * R * (K + N)}
    T, top, E = case["T"], case["top"], case["E"]
    n = T * top
    used = min(E, n)
    if op == "experts":
        N, K = case["N"], case["K"]
        b, f = _entry_bytes(N, K, case["split"], case["dense_frac"])
        k = 2 if case["pair"] else 1
        return {"bytes": k * (used * (b + 4 * N) + 2 * n * N) + T * (K + 4) + 8 * n, "flops": 2 * k * n * f}
    H, I = case["hidden"], case["inter"]
    b1, f1 = _entry_bytes(I, H, "output", case["dense_frac"])
    b2, f2 = _entry_bytes(H, I, "input", case["dense_frac"])
    return {"bytes": used * (2 * b1 + b2 + 8 * I + 4 * H) + T * (H + 4) + 2 * T * H + 8 * n,
            "flops": 2 * n * (2 * f1 + f2)}
