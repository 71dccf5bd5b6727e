"""Measured cases of the operators around tree attention: normalised and rotated heads placed into the cache, attention
with capped or distance-biased scores, sampled tokens and sampled verification -- with their plain forms in torch.

``run`` computes an operator in its plain form (32-bit arithmetic, 64 bits for angles, for probabilities and for their
sums) or, with ``own`` set, through this package's entry points.  ``exact`` restates the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ZERO_WEIGHT_LOG2 = -1000.0        # a token whose weight relative to the most likely one is below 2^-1000 counts as zero


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def _place(name, B, N, Hq, Hkv, D, dtype, kv, page, rot, interleaved, scaling):
    return {"name": name, "op": "place", "B": B, "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "kv": kv, "page": page,
            "rot": rot, "interleaved": interleaved, "scaling": scaling}


def _attend(name, B, N, Hq, Hkv, D, dtype, lo, hi, page, cap, bias):
    return {"name": name, "op": "attend", "B": B, "N": N, "Hq": Hq, "Hkv": Hkv, "D": D, "dtype": dtype, "kv_lo": lo, "kv_hi": hi,
            "page": page, "cap": cap, "bias": bias}


def _sample(name, B, N, V, dtype, top_k, top_p, min_p, spread):
    return {"name": name, "op": "sample", "B": B, "N": N, "V": V, "dtype": dtype, "top_k": top_k, "top_p": top_p, "min_p": min_p,
            "spread": spread}


def _verify(name, B, T, pseudo, V, dtype, top_k, top_p, min_p, spread):
    return {"name": name, "op": "verify", "B": B, "T": T, "N": T + pseudo, "V": V, "dtype": dtype, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "spread": spread}


def listed():
    return [
        # one sequence's 88 tree nodes and 3 pseudo rows: the latency of a single decoding round
        _place("place_1x91_f16", 1, 91, 32, 32, 128, "f16", 1024, 0, 128, False, "none"),
        # four sequences on a paged cache; only half of each head is rotated, neighbouring features paired
        _place("place_4x91_paged_partial", 4, 91, 32, 32, 128, "bf16", 4096, 64, 64, True, "linear"),
        # prompts of grouped-query heads far into a scaled context: bandwidth
        _place("place_8x2048_prompt", 8, 2048, 64, 8, 128, "bf16", 0, 0, 128, False, "parts"),
        # the smallest shape of this repository: fp32, heads of 64, on the ALU kernel
        _attend("attend_tiny_f32_both", 1, 18, 4, 4, 64, "f32", 128, 128, 0, 30.0, True),
        # one sequence of 1024 keys, capped scores
        _attend("attend_1x91_kv1024_cap", 1, 91, 32, 32, 128, "f16", 1024, 1024, 0, 50.0, False),
        # ragged lengths, capped scores and a distance bias together
        _attend("attend_8x68_ragged_both", 8, 68, 40, 40, 128, "bf16", 512, 8192, 0, 30.0, True),
        # grouped heads on a paged cache with a distance bias: the tile-pair kernel, large batch
        _attend("attend_16x67_paged_bias", 16, 67, 64, 8, 128, "bf16", 8192, 8192, 64, 0.0, True),
        # the next token of four sequences, the filters most servers set
        _sample("sample_4_32000_top_k_p", 4, 1, 32000, "bf16", 50, 0.95, 0.0, 2.5),
        # a larger vocabulary in 32 bits, nucleus and minimum probability, a full batch
        _sample("sample_64_131072_top_p", 64, 1, 131072, "f32", 0, 0.9, 0.02, 2.5),
        # odd vocabulary, no filters, flat distributions: the whole row counts
        _sample("sample_256_32003_plain", 256, 1, 32003, "f16", 0, 1.0, 0.0, 1.0),
        # verification of one sequence's 88 nodes
        _verify("verify_1x88_top_k_p", 1, 88, 3, 32000, "f16", 40, 0.95, 0.0, 2.5),
        # sixteen sequences of 256 nodes
        _verify("verify_16x256_top_p", 16, 256, 3, 32000, "bf16", 0, 0.95, 0.0, 2.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["place", "attend", "sample", "verify"])
    dtype = rng.choice(["f16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 32, 40])
    group = rng.choice([1, 1, 2, 4, 8]) if Hkv <= 8 else 1
    if op == "place":
        B = _log_int(rng, 1, 16)
        N = _log_int(rng, 1, max(1, 8 * 2048 * 80 // (B * (group + 2) * Hkv * (2 if dtype == "f32" else 1)) if Hkv >= 8 else 1024))
        N = min(N, 2048)
        interleaved = rng.random() < 0.5
        rot = rng.choice([D, D, D // 2, D // 4]) if not interleaved else rng.choice([D, D // 2, 2 * rng.randint(1, D // 2)])
        return {k: v for k, v in _place("", B, N, group * Hkv, Hkv, D, dtype, _log_int(rng, 1, 2048), rng.choice([0, 0, 16, 64, 128]), rot,
                                        interleaved, rng.choice(["none", "linear", "parts"])).items() if k != "name"}
    if op == "attend":
        small = dtype == "f32" or D == 64                      # the ALU kernel's range
        B, N = _log_int(rng, 1, 4 if small else 16), _log_int(rng, 1, 24 if small else 260)
        room = (24 << 20) if small else (16 * 67 * 64 * 8192)
        hi = max(16, min(512 if small else 8192, room // (B * N * group * Hkv)))
        hi = _log_int(rng, 16, hi)
        page = 0 if small else rng.choice([0, 0, 16, 64, 128])
        cap, bias = rng.choice([(0.0, True), (30.0, False), (50.0, False), (30.0, True), (rng.uniform(5.0, 80.0), True)])
        return {k: v for k, v in _attend("", B, N, group * Hkv, Hkv, D, dtype, max(1, hi // rng.choice([1, 2, 16])), hi, page, cap,
                                         bias).items() if k != "name"}
    filters = rng.choice([(0, 1.0, 0.0), (0, rng.uniform(0.5, 0.99), 0.0), (_log_int(rng, 1, 2000), 1.0, 0.0),
                          (_log_int(rng, 2, 200), rng.uniform(0.5, 0.99), 0.0), (0, 1.0, rng.uniform(0.001, 0.2)),
                          (_log_int(rng, 2, 20000), rng.uniform(0.8, 0.99), rng.uniform(0.001, 0.1))])
    V = _log_int(rng, 500, 160000)
    if op == "sample":
        B = _log_int(rng, 1, min(256, max(1, (32 << 20) // V)))
        return {k: v for k, v in _sample("", B, 1, V, dtype, *filters, rng.uniform(0.8, 4.0)).items() if k != "name"}
    B = _log_int(rng, 1, 16)
    T = _log_int(rng, 1, min(256, max(1, (64 << 20) // (V * B))))
    return {k: v for k, v in _verify("", B, T, rng.randint(0, 4), V, dtype, *filters, rng.uniform(0.8, 4.0)).items() if k != "name"}


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
SCALING = {"none": {}, "linear": {"factor": 4.0}, "parts": {"factor": 8.0, "low": 1.0, "high": 4.0, "orig_len": 8192, "magnitude": 1.0}}


def _trees(rng, B, T, N):
    """Random draft trees of depth at most 6 and, behind them, a chain of pseudo rows hanging off one node."""
    parent = np.full((B, N), -1, np.int32)
    depth = np.zeros((B, N), np.int64)
    for b in range(B):
        for r in range(1, T):
            allowed = np.flatnonzero(depth[b, :r] < 5)
            parent[b, r] = rng.choice(allowed)
            depth[b, r] = depth[b, parent[b, r]] + 1
        for r in range(T, N):
            parent[b, r] = rng.integers(0, T) if r == T else r - 1
            depth[b, r] = depth[b, parent[b, r]] + 1
    return parent, depth


def _pool(flat, table, page):
    """A contiguous cache [B, H, cap, D] as a pool of pages [n, H, page, D] under `table` [B, cap / page]."""
    B, H, cap, D = flat.shape
    pool = torch.empty((int(table.numel()) + 1, H, page, D), dtype=flat.dtype, device=flat.device)
    pool[table.long().flatten()] = flat.view(B, H, cap // page, page, D).permute(0, 2, 1, 3, 4).reshape(-1, H, page, D)
    pool[-1] = 0
    return pool


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = DTYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    dev = lambda a, t=torch.int32: torch.as_tensor(a, dtype=t).cuda()       # noqa: E731
    B, N = case["B"], case["N"]
    st = {"case": case, "B": B, "N": N}
    if case["op"] in ("sample", "verify"):
        V = case["V"]
        logits = normal(B, N, V).mul_(case["spread"])
        likely = torch.randint(0, V, (B, N), generator=g, device="cuda")
        # the confident rows of a model: one token some way above the rest (not in the flat case)
        boost = torch.rand((B, N), generator=g, device="cuda") * (6.0 * case["spread"] if case["spread"] > 1.0 else 0.0)
        logits.scatter_add_(2, likely[..., None], boost[..., None])
        st["logits"] = logits.to(dt)
        st["uniform"] = torch.rand((B, N), generator=g, device="cuda")
        st["temperature"] = torch.rand(B, generator=g, device="cuda") * 0.9 + 0.3
        st["top_k"] = torch.full((B,), case["top_k"], dtype=torch.int32, device="cuda") if case["top_k"] else None
        st["top_p"] = torch.full((B,), case["top_p"], device="cuda") if case["top_p"] < 1.0 else None
        st["min_p"] = torch.full((B,), case["min_p"], device="cuda") if case["min_p"] > 0.0 else None
        if case["op"] == "verify":
            T = case["T"]
            parent, _ = _trees(rng, B, T, N)
            st["parent"] = dev(parent)
            tokens = torch.randint(0, V, (B, T), generator=g, device="cuda")
            first_child = np.zeros((B, T), bool)
            for b in range(B):
                first_child[b, 1:] = [p not in parent[b, 1:r] for r, p in enumerate(parent[b, 1:T], 1)]
            from_parent = torch.gather(likely, 1, dev(parent[:, :T].clip(0), torch.int64))
            st["tokens"] = torch.where(dev(first_child, torch.bool), from_parent, tokens).int()
            st["root_pred"] = st["tokens"][:, 0].clone().contiguous()
            st["max_path"] = 8
            st["accept_len"] = torch.zeros(B, dtype=torch.int32, device="cuda")
        return st
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    if case["op"] == "place":
        lens = np.full(B, case["kv"])
        # the rows as a fused projection leaves them: q, k and v side by side
        qkv = normal(B, N, (Hq + 2 * Hkv) * D).to(dt)
        st["q"] = qkv[..., :Hq * D].unflatten(2, (Hq, D))
        st["k"] = qkv[..., Hq * D:(Hq + Hkv) * D].unflatten(2, (Hkv, D))
        st["v"] = qkv[..., (Hq + Hkv) * D:].unflatten(2, (Hkv, D))
        st["q_weight"], st["k_weight"] = (1 + 0.2 * normal(D)).to(dt), (1 + 0.2 * normal(D)).to(dt)
        far = rng.integers(0, 100000, (B, 1))
        st["pos"] = dev(far + (np.arange(N)[None] if N > 512 else rng.integers(0, 8, (B, N))))
        st["q_out"] = torch.empty((B, N, Hq, D), dtype=dt, device="cuda")
        st["base"], st["eps"] = 500000.0, 1e-6
    else:
        lens = rng.integers(case["kv_lo"], case["kv_hi"] + 1, B)
        T = max(1, N - 3)
        parent, depth = _trees(rng, B, T, N)
        st["parent"], st["pos"] = dev(parent), dev(lens[:, None] + depth)
        st["q"] = normal(B, N, Hq, D).mul_(3.0).to(dt)
        st["slopes"] = dev(2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq), torch.float32) if case["bias"] else None
        st["out"] = torch.empty_like(st["q"])
        # kept between calls by a program, as zeros once
        st["workspace"] = torch.zeros(48 << 20, dtype=torch.uint8, device="cuda")
    unit = page if page else 16
    cap = (int(lens.max()) + N + unit - 1) // unit * unit
    k, v = normal(B, Hkv, cap, D).to(dt), normal(B, Hkv, cap, D).to(dt)
    st["kv_len"], st["top"] = dev(lens), int(lens.max()) + N
    if page:
        st["table"] = dev(rng.permutation(B * (cap // page)).reshape(B, cap // page))
        k, v = _pool(k, st["table"], page), _pool(v, st["table"], page)
    st["k_cache"], st["v_cache"] = k, v
    return st


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _frequencies(st, device):
    """Angles per position of the rotated pairs, in 64 bits."""
    case = st["case"]
    rot, how, s = case["rot"], case["scaling"], SCALING[case["scaling"]]
    f = st["base"] ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device=device) / rot)
    if how == "linear":
        return f / s["factor"]
    if how == "parts":
        turns = s["orig_len"] * f / (2 * math.pi)
        keep = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0, 1)
        return f * (keep + (1 - keep) / s["factor"])
    return f


def _heads_plain(x, weight, st):
    """RMS norm of each head, then the rotation of its first `rot` features: 32 bits throughout."""
    rot = st["case"]["rot"]
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + st["eps"]) * weight.float()
    angle = (st["pos"].double()[..., None] * _frequencies(st, x.device))[:, :, None]
    cos, sin = angle.cos().float(), angle.sin().float()
    head, rest = y[..., :rot], y[..., rot:]
    if st["case"]["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        head = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((head, rest), -1).to(x.dtype)


def _place_plain(st):
    B, N, page = st["B"], st["N"], st["case"]["page"]
    st["q_out"].copy_(_heads_plain(st["q"], st["q_weight"], st))
    k = _heads_plain(st["k"], st["k_weight"], st)
    row = st["kv_len"].long()[:, None] + torch.arange(N, device=k.device)
    if page:
        at, row = torch.gather(st["table"].long(), 1, row // page), row % page
    else:
        at = torch.arange(B, device=k.device)[:, None].expand(B, N)
    st["k_cache"][at, :, row] = k
    st["v_cache"][at, :, row] = st["v"]
    return st["q_out"], st["k_cache"], st["v_cache"], torch.zeros(B, dtype=torch.int32, device=k.device)


def _ancestors(parent):
    """[B, N, N] truth values: is c row r itself or an ancestor of it?"""
    N = parent.shape[1]
    step = torch.nn.functional.one_hot(parent.long() + 1, N + 1)[..., 1:].double() + torch.eye(N, dtype=torch.float64, device=parent.device)
    return torch.linalg.matrix_power(step, N) > 0


def _rows_of(cache, st):
    if not st["case"]["page"]:
        return cache[:, :, :st["top"]]
    return cache[st["table"].long()].permute(0, 2, 1, 3, 4).flatten(2, 3)[:, :, :st["top"]]


def _attend_plain(st):
    case, q = st["case"], st["q"]
    B, N, Hq, D = q.shape
    Hkv, cap, top = case["Hkv"], case["cap"], st["top"]
    k, v = _rows_of(st["k_cache"], st).float(), _rows_of(st["v_cache"], st).float()
    rows = q.float().view(B, N, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, D)
    s = (rows @ k.transpose(-1, -2)).mul_(D ** -0.5).view(B, Hkv, Hq // Hkv, N, top)
    if cap:
        s = s.div_(cap).tanh_().mul_(cap)
    key = torch.arange(top, device=q.device)
    node = key - st["kv_len"][:, None]                                                 # [B, top]: index among the tree rows
    inside = node.clamp(0, N - 1).long()
    if case["bias"]:
        key_pos = torch.where(node < 0, key, torch.gather(st["pos"], 1, inside))
        away = (st["pos"][:, :, None] - key_pos[:, None]).float()                      # [B, N, top]
        s -= st["slopes"].view(1, Hkv, Hq // Hkv, 1, 1) * away[:, None, None]
    seen = torch.gather(_ancestors(st["parent"]), 2, inside[:, None].expand(B, N, top)) & (node < N)[:, None] | (node < 0)[:, None]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    p = (s - s.amax(-1, keepdim=True)).exp_()
    p = p / p.sum(-1, keepdim=True)
    v = v.masked_fill((node >= N)[:, None, :, None], 0.0)                                # cache rows behind the tree are not data
    out = p.flatten(2, 3) @ v
    st["out"].copy_(out.view(B, Hkv, Hq // Hkv, N, D).permute(0, 3, 1, 2, 4).reshape(B, N, Hq, D))
    return st["out"], torch.zeros(B, dtype=torch.int32, device=q.device)


def _sample_plain(st, logits, uniform):
    """One token per row [B, R]: weights relative to the most likely token, filters along the order (larger logit first,
    lower index among equals), the first kept token in index order whose running sum exceeds uniform * total."""
    B, R, V = logits.shape
    x = logits.float()
    x = x.masked_fill(x.isnan(), -math.inf)
    value, index = x.sort(dim=-1, descending=True, stable=True)
    per_row = lambda t: t.view(B, 1, 1)                                                 # noqa: E731
    gap = torch.where(value == value[..., :1], 0.0, value.double() - value[..., :1].double())
    power = gap / per_row(st["temperature"]).double()
    w = power.exp().masked_fill_(power < ZERO_WEIGHT_LOG2 * math.log(2.0), 0.0)
    place = torch.arange(V, device=x.device)
    keep = torch.ones_like(w, dtype=torch.bool)
    if st["top_k"] is not None:
        k = per_row(st["top_k"])
        keep &= (place < k) | (k <= 0)
    if st["top_p"] is not None:
        p = per_row(st["top_p"]).double()
        kept = w * keep
        running = kept.cumsum(-1)
        before = torch.cat((torch.zeros_like(running[..., :1]), running[..., :-1]), -1)
        keep &= (before < p * running[..., -1:]) | (p >= 1.0) | (place == 0)
    if st["min_p"] is not None:
        keep &= w >= per_row(st["min_p"]).double()
    w = torch.zeros_like(w).scatter_(-1, index, w * keep)
    running = w.cumsum(-1)
    past = (running > uniform[..., None].double() * running[..., -1:]) & (w > 0)
    last = (V - 1 - (w > 0).flip(-1).to(torch.int8).argmax(-1))
    return torch.where(past.any(-1), past.to(torch.int8).argmax(-1), last).int()


def _verify_plain(st):
    T, N, B = st["case"]["T"], st["N"], st["B"]
    dev = st["logits"].device
    pred = torch.full((B, N), -1, dtype=torch.int32, device=dev)
    pred[:, :T] = _sample_plain(st, st["logits"][:, :T], st["uniform"][:, :T])
    par = st["parent"][:, :T].long()
    line = _ancestors(st["parent"][:, :T])                                             # [B, node, ancestor or self]
    expected = torch.where(par < 0, st["root_pred"][:, None], torch.gather(pred, 1, par.clamp(min=0)))
    good = ~(line & (st["tokens"] != expected)[:, None]).any(-1)
    depth = line.sum(-1)
    node = torch.arange(T, device=dev)
    key = torch.where(good, depth * (T + 1) + (T - node), 0)
    best = key.argmax(-1)
    length = torch.where(good.any(-1), torch.gather(depth, 1, best[:, None])[:, 0], 0)
    on_path = torch.gather(line, 1, best[:, None, None].expand(B, 1, T))[:, 0] & (length > 0)[:, None]
    path = torch.where(on_path, node, T).sort(-1).values
    path = torch.nn.functional.pad(path, (0, st["max_path"]), value=T)[:, :st["max_path"]]
    path = torch.where(path < T, path, -1).int()
    last = torch.where(length > 0, torch.gather(pred, 1, best[:, None])[:, 0], st["root_pred"])
    return pred, length.int(), path, last, torch.zeros(B, dtype=torch.int32, device=dev)


# ---------------------------------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------------------------------
def run(state):
    st, case = state, state["case"]
    op = case["op"]
    if not own:
        if op == "place":
            return _place_plain(st)
        if op == "attend":
            return _attend_plain(st)
        if op == "sample":
            return _sample_plain(st, st["logits"], st["uniform"]), torch.zeros(st["B"], dtype=torch.int32, device="cuda")
        return _verify_plain(st)
    from paper_2404_12022_b200 import binding as hb
    if op == "place":
        how = {"none": hb.HT_ROPE_PLAIN, "linear": hb.HT_ROPE_LINEAR, "parts": hb.HT_ROPE_BY_PARTS}[case["scaling"]]
        head = hb.make_head_desc(case["D"], eps=st["eps"], rot_dim=case["rot"], interleaved=case["interleaved"], rope_base=st["base"],
                                 scaling=how, **SCALING[case["scaling"]])
        if case["page"]:
            q, status = hb.norm_rope_kv_append_paged(st["q"], st["k"], st["v"], st["pos"], st["kv_len"], st["table"], st["k_cache"],
                                                     st["v_cache"], head, st["q_weight"], st["k_weight"], q_out=st["q_out"])
        else:
            q, status = hb.norm_rope_kv_append(st["q"], st["k"], st["v"], st["pos"], st["kv_len"], st["k_cache"], st["v_cache"], head,
                                               st["q_weight"], st["k_weight"], q_out=st["q_out"])
        return q, st["k_cache"], st["v_cache"], status
    if op == "attend":
        kw = dict(cap=case["cap"], slopes=st["slopes"], pos=st["pos"], out=st["out"], workspace=st["workspace"],
                  flags=hb.HT_ATTN_WORKSPACE_CLEAN)
        if case["page"]:
            return hb.tree_attention_scored_paged(st["q"], st["k_cache"], st["v_cache"], st["table"], st["kv_len"], st["parent"], **kw)
        return hb.tree_attention_scored(st["q"], st["k_cache"], st["v_cache"], st["kv_len"], st["parent"], **kw)
    filters = dict(temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
    if op == "sample":
        return hb.sample(st["logits"], st["uniform"], **filters)
    return hb.verify_sampled(st["logits"], st["uniform"], st["tokens"], st["parent"], st["root_pred"], max_path=st["max_path"],
                             accept_len=st["accept_len"], **filters)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    B, N = case["B"], case["N"]
    if case["op"] in ("sample", "verify"):
        rows = B * case.get("T", N)
        return {"bytes": rows * case["V"] * e + 8 * rows, "flops": 4 * rows * case["V"]}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "place":
        values = B * N * (Hq + 2 * Hkv) * D
        return {"bytes": 2 * values * e + 4 * B * N, "flops": 8 * values}
    keys = (case["kv_lo"] + case["kv_hi"]) // 2 + N
    return {"bytes": e * D * (2 * B * Hkv * keys + 2 * B * N * Hq), "flops": 4 * B * N * Hq * keys * D}


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _np(t):
    return None if t is None else (t.double() if t.is_floating_point() else t).cpu().numpy()


def _exact_heads(x, weight, pos, st):
    case, rot = st["case"], st["case"]["rot"]
    s = SCALING[case["scaling"]]
    x = x.double()
    y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + st["eps"]) * weight.double()
    out = y.clone()
    for i in range(rot // 2):
        f = math.exp(-2.0 * i / rot * math.log(st["base"]))
        if case["scaling"] == "linear":
            f /= s["factor"]
        elif case["scaling"] == "parts":
            wavelength = 2 * math.pi / f
            mix = min(1.0, max(0.0, (s["orig_len"] / wavelength - s["low"]) / (s["high"] - s["low"])))
            f = (1 - mix) * f / s["factor"] + mix * f
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
        c, d = torch.cos(pos.double() * f)[..., None], torch.sin(pos.double() * f)[..., None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * d, y[..., a] * d + y[..., b] * c
    return out


def _exact_place(st):
    B, N, page = st["B"], st["N"], st["case"]["page"]
    q = _exact_heads(st["q"], st["q_weight"], st["pos"], st)
    k = _exact_heads(st["k"], st["k_weight"], st["pos"], st)
    kc, vc = st["k_cache"].double(), st["v_cache"].double()
    table = _np(st["table"]) if page else None
    for b, L in enumerate(st["kv_len"].tolist()):
        for r in range(N):
            at, row = (int(table[b, (L + r) // page]), (L + r) % page) if page else (b, L + r)
            kc[at, :, row], vc[at, :, row] = k[b, r], st["v"][b, r].double()
    return q, kc, vc, torch.zeros(B, dtype=torch.int32)


def _exact_attend(st):
    case, q = st["case"], st["q"].double()
    B, N, Hq, D = q.shape
    out = torch.empty_like(q)
    parent, lens = st["parent"].cpu().numpy(), st["kv_len"].tolist()
    for b in range(B):
        L = lens[b]
        seen = np.zeros((N, L + N), bool)
        for r in range(N):
            seen[r, :L], seen[r, L + r] = True, True
            if parent[b, r] >= 0:
                seen[r, L:] |= seen[parent[b, r], L:]
        seen = torch.from_numpy(seen).cuda()
        at = torch.cat((torch.arange(L, device="cuda"), st["pos"][b].long()))
        away = (st["pos"][b].long()[:, None] - at).double()
        rows = torch.arange(L + N, device="cuda")
        for h in range(Hq):
            kv = h // (Hq // case["Hkv"])
            if case["page"]:
                page = st["table"][b].long()[rows // case["page"]]
                k, v = (c[page, kv, rows % case["page"]].double() for c in (st["k_cache"], st["v_cache"]))
            else:
                k, v = (c[b, kv, :L + N].double() for c in (st["k_cache"], st["v_cache"]))
            s = q[b, :, h] @ k.T / math.sqrt(D)
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            if case["bias"]:
                s = s - float(st["slopes"][h]) * away
            out[b, :, h] = torch.softmax(torch.where(seen, s, -math.inf), -1) @ v
    return out, torch.zeros(B, dtype=torch.int32)


def _exact_token(x, u, T, k, p, floor):
    """One row, by the definition: x float64 logits without NaN."""
    order = np.lexsort((np.arange(x.size), -x))
    gap = np.where(x[order] == x[order[0]], 0.0, x[order] - x[order[0]]) / T
    w = np.where(gap < ZERO_WEIGHT_LOG2 * np.log(2.0), 0.0, np.exp(gap))
    n = x.size if not k or k <= 0 else min(int(k), x.size)
    if p is not None and p < 1.0:
        running = np.cumsum(w[:n])
        n = max(1, int(np.searchsorted(np.concatenate(([0.0], running[:-1])), p * running[-1], side="left")))
    if floor is not None:
        n = min(n, int(np.count_nonzero(w >= floor)))
    n = min(n, int(np.count_nonzero(w > 0)))
    ids = np.sort(order[:n])
    weight = np.zeros(x.size)
    weight[order[:n]] = w[:n]
    running = np.cumsum(weight[ids])
    j = int(np.searchsorted(running, u * running[-1], side="right"))
    return int(ids[min(j, n - 1)])


def _exact_tokens(st, R):
    x = _np(st["logits"][:, :R])
    x = np.where(np.isnan(x), -np.inf, x)
    u, T, k, p, m = (_np(st[name]) for name in ("uniform", "temperature", "top_k", "top_p", "min_p"))
    at = lambda a, b: None if a is None else a[b]                                       # noqa: E731
    return np.array([[_exact_token(x[b, r], u[b, r], T[b], at(k, b), at(p, b), at(m, b)) for r in range(R)] for b in range(st["B"])], np.int32)


def _exact_verify(st):
    B, T, N = st["B"], st["case"]["T"], st["N"]
    pred = np.full((B, N), -1, np.int32)
    pred[:, :T] = _exact_tokens(st, T)
    tokens, parent, root = st["tokens"].cpu().numpy(), st["parent"].cpu().numpy(), st["root_pred"].cpu().numpy()
    length, path, last = np.zeros(B, np.int32), np.full((B, st["max_path"]), -1, np.int32), root.copy()
    for b in range(B):
        best = []
        reached = {}
        for n in range(T):
            p = parent[b, n]
            if tokens[b, n] == (root[b] if p < 0 else pred[b, p]) and (p < 0 or p in reached):
                reached[n] = (reached[p] if p >= 0 else []) + [n]
                best = reached[n] if len(reached[n]) > len(best) else best
        length[b] = len(best)
        path[b, :len(best)] = best
        last[b] = pred[b, best[-1]] if best else root[b]
    return tuple(torch.from_numpy(a) for a in (pred, length, path, last, np.zeros(B, np.int32)))


def exact(case, seed):
    if case["op"] in ("sample", "verify") and case["B"] * case.get("T", case["N"]) * case["V"] > 40_000_000:
        return None
    st = prepare(case, seed)
    if case["op"] == "place":
        return _exact_place(st)
    if case["op"] == "attend":
        return _exact_attend(st)
    if case["op"] == "sample":
        return torch.from_numpy(_exact_tokens(st, case["N"])), torch.zeros(case["B"], dtype=torch.int32)
    return _exact_verify(st)
