"""Operators around the compressed cache, as a serving program calls them: rotary positions on the way
into the cache, attention of whole prompts, attention of drafted token trees, and the accepted path's
way into the cache.

Four kinds of pass, each one call of the public binding:

``rotary``  packed tokens' Q, K and V -> rotated queries, rotated keys and values in their slots, norms, ids
``prompt``  causal attention of packed sequences, over their own rows or over a cache that ends with them
``tree``    attention of drafted nodes over a slot cache and, as a mask allows, over one another
``path``    rows of the accepted nodes of every layer appended to the slot cache

``own`` False computes the same in elementary torch operations.  Keys follow the recipe of
``paper_2406_11430_amd/synth.py``: rows ``s*g``, ``g ~ N(0,1)``, ``s = exp(z/2)``, with a few low-norm
tokens at the start of every sequence; values and queries ``N(0,1)``.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SINK_TOKENS, SINK_SCALE = 4, 0.1
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3}


# ---------------------------------------------------------------------------- the cases
def listed():
    return [
        # one decode step of a batch: a token for each of 64 sequences, fp32, part of every head rotated
        {"name": "rotary_step_f32", "kind": "rotary", "dtype": "f32", "n_seq": 64, "packed": False, "new_lo": 1,
         "new_hi": 1, "have_lo": 490, "have_hi": 4096, "Hq": 8, "Hkv": 4, "D": 64, "rot": 32,
         "layout": "interleaved", "scaling": "linear"},
        # the prompts of a ragged batch, straight from the projection: packed, whole heads, far positions
        {"name": "rotary_prompts", "kind": "rotary", "dtype": "bf16", "n_seq": 8, "new_lo": 1000, "new_hi": 8192,
         "packed": True, "Hq": 32, "Hkv": 8, "D": 128, "rot": 128, "layout": "half", "scaling": "bands"},
        # the shortest prompt: launches are all there is
        {"name": "prompt_short", "kind": "prompt", "dtype": "bf16", "n_seq": 1, "new_lo": 37, "new_hi": 37,
         "have_lo": 0, "have_hi": 0, "Hq": 32, "Hkv": 8, "D": 128},
        # a ragged batch of prompts, 1k to 8k tokens
        {"name": "prompt_packed", "kind": "prompt", "dtype": "bf16", "n_seq": 16, "new_lo": 1024, "new_hi": 8192,
         "have_lo": 0, "have_hi": 0, "Hq": 32, "Hkv": 8, "D": 128},
        # one prompt of 32k tokens: the largest
        {"name": "prompt_32k", "kind": "prompt", "dtype": "bf16", "n_seq": 1, "new_lo": 32768, "new_hi": 32768,
         "have_lo": 0, "have_hi": 0, "Hq": 32, "Hkv": 8, "D": 128},
        # the next turn of four conversations over their compressed caches
        {"name": "prompt_turn_over_cache", "kind": "prompt", "dtype": "bf16", "n_seq": 4, "new_lo": 100,
         "new_hi": 301, "have_lo": 13108, "have_hi": 16384, "Hq": 32, "Hkv": 8, "D": 128},
        # fp32 model of the toy size's rows, odd lengths, no grouping
        {"name": "prompt_odd_f32", "kind": "prompt", "dtype": "f32", "n_seq": 3, "new_lo": 511, "new_hi": 1533,
         "have_lo": 0, "have_hi": 77, "Hq": 4, "Hkv": 4, "D": 64},
        # a few drafted tokens over a short cache: latency
        {"name": "tree_small", "kind": "tree", "dtype": "bf16", "n_seq": 1, "nodes_lo": 7, "nodes_hi": 7,
         "have_lo": 2048, "have_hi": 2048, "Hq": 32, "Hkv": 32, "D": 128},
        # the streaming batch with trees of up to 32 drafted nodes over caches at half their prompts
        {"name": "tree_batch", "kind": "tree", "dtype": "bf16", "n_seq": 64, "nodes_lo": 1, "nodes_hi": 32,
         "have_lo": 500, "have_hi": 4000, "Hq": 32, "Hkv": 8, "D": 128},
        # 63 nodes over an uncompressed layer of 131k tokens
        {"name": "tree_131k", "kind": "tree", "dtype": "bf16", "n_seq": 1, "nodes_lo": 63, "nodes_hi": 63,
         "have_lo": 131072, "have_hi": 131072, "Hq": 32, "Hkv": 8, "D": 128},
        # accepted tokens of one fp32 sequence
        {"name": "path_one_f32", "kind": "path", "dtype": "f32", "L": 2, "n_seq": 1, "nodes_lo": 9, "nodes_hi": 9,
         "path_lo": 3, "path_hi": 3, "have_lo": 777, "have_hi": 777, "Hkv": 4, "D": 64},
        # accepted tokens of the streaming batch, eight layers
        {"name": "path_batch", "kind": "path", "dtype": "bf16", "L": 8, "n_seq": 64, "nodes_lo": 1, "nodes_hi": 64,
         "path_lo": 1, "path_hi": 9, "have_lo": 256, "have_hi": 512, "Hkv": 8, "D": 128},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, what, lo, hi):
    a, b = sorted((_log_int(rng, lo, hi), _log_int(rng, lo, hi)))
    return {what + "_lo": a, what + "_hi": b}


# rows the library supports, and the largest query group of each
ROWS = [("bf16", 128, 8), ("bf16", 64, 8), ("bf16", 256, 4), ("f32", 128, 8), ("f32", 64, 8)]


def draw(rng):
    kind = rng.choice(["rotary", "prompt", "prompt", "tree", "tree", "path"])
    dtype, D, most = rng.choice(ROWS + ROWS[:1] * 3)
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([g for g in (1, 2, 3, 4, 7, 8) if g <= most])
    case = {"kind": kind, "dtype": dtype, "Hkv": Hkv, "D": D}
    if kind != "path":
        case["Hq"] = Hkv * G
    if kind == "rotary":
        n_seq = _log_int(rng, 1, 64)
        packed = rng.random() < 0.5
        case.update(n_seq=n_seq, packed=packed, **_span(rng, "new", 1, max(2, 32768 // n_seq)), **_span(rng, "have", 1, 4096),
                    rot=rng.choice([r for r in (16, 32, 48, 64, 96, 128, 256) if r <= D]), layout=rng.choice(list(LAYOUTS)),
                    scaling=rng.choice(list(SCALINGS)))
    elif kind == "prompt":
        n_seq = _log_int(rng, 1, 16)
        top = (8192 if dtype == "bf16" else 2048) // (1 if n_seq < 4 else 2)
        fresh = rng.random() < 0.5
        case.update(n_seq=n_seq, **_span(rng, "new", 1, top), **_span(rng, "have", 1, 16384 // n_seq))
        if fresh:
            case.update(have_lo=0, have_hi=0)
    elif kind == "tree":
        n_seq = _log_int(rng, 1, 64)
        case.update(n_seq=n_seq, **_span(rng, "nodes", 1, 64), **_span(rng, "have", 1, 65536 // n_seq))
    else:
        case.update(L=rng.choice([1, 2, 5, 8]), n_seq=_log_int(rng, 1, 64), **_span(rng, "nodes", 1, 64), **_span(rng, "path", 1, 12),
                    **_span(rng, "have", 1, 512))
    return case


def _spread(case, what):
    """One length for each sequence, evenly over the case's range, in an order that does not rise."""
    lo, hi, n = case[what + "_lo"], case[what + "_hi"], case["n_seq"]
    step = next(s for s in (7, 5, 3, 11, 1) if math.gcd(s, n) == 1)
    return [hi if n == 1 else lo + (hi - lo) * ((i * step + n // 2) % n) // (n - 1) for i in range(n)]


def _starts(lens):
    out = [0]
    for x in lens:
        out.append(out[-1] + x)
    return out


# ---------------------------------------------------------------------------- inputs
def _keys(gen, heads, lens, D):
    """[heads, sum(lens), D] fp32 by the recipe of the synthetic caches."""
    total = sum(lens)
    k = torch.randn((heads, total, D), generator=gen, device="cuda")
    k *= torch.exp(0.5 * torch.randn((heads, total, 1), generator=gen, device="cuda"))
    for start, n in zip(_starts(lens), lens):
        k[:, start:start + min(SINK_TOKENS, n)] *= SINK_SCALE
    return k


def _dev(values, dtype):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _frequencies(case):
    """Angle per position of every pair, double.  bands: pairs that turn more than `high` times over the original
    context stay, those that turn less than `low` times are slowed down by the factor, a ramp lies between."""
    R = case["rot"]
    base, factor, original, low, high = 500000.0, 8.0, 8192, 1.0, 4.0
    if own:
        import paper_2406_11430_amd as l2kv
        return l2kv.l2kv_rotary_freqs(R, base, SCALINGS[case["scaling"]], factor, original, low, high).cuda()
    i = torch.arange(R // 2, dtype=torch.float64)
    if case["scaling"] == "base":
        base = base * factor ** (R / (R - 2))
    f = base ** (-2.0 * i / R)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "bands":
        turns = original * f / (2 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f.cuda()


def _tree_masks(gen_cpu, nodes, words):
    """Random trees: node i's parent is one of the nodes before it (the first is a root); bit j of row i where j is i or above it."""
    rows = []
    for n in nodes:
        for i in range(n):
            mask = 1 << i
            if i > 0:
                parent = int(torch.randint(max(0, i - 6), i, (1,), generator=gen_cpu))
                mask |= rows[len(rows) - i + parent]
            rows.append(mask)
    out = torch.tensor([[(m >> (32 * w)) & 0xffffffff for w in range(words)] for m in rows], dtype=torch.int64)
    return torch.where(out >= 1 << 31, out - (1 << 32), out).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    gen_cpu = torch.Generator().manual_seed(seed)
    kind, dt, D, Hkv = case["kind"], DTYPES[case["dtype"]], case["D"], case["Hkv"]
    st = {"case": case, "kind": kind}
    if kind == "rotary":
        new, Hq = _spread(case, "new"), case["Hq"]
        total = sum(new)
        # the projection's output: queries, keys and values of a token side by side
        qkv = torch.randn((total, Hq + 2 * Hkv, D), generator=gen, device="cuda")
        qkv[:, Hq:Hq + Hkv] *= torch.exp(0.5 * torch.randn((total, Hkv, 1), generator=gen, device="cuda"))
        qkv = qkv.to(dt)
        st["Q"], st["K"], st["V"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        packed = case["packed"]                                        # no cache before: rows where the tokens are
        have = [0] * case["n_seq"] if packed else _spread(case, "have")
        # a cache that has dropped tokens: positions run ahead of slots
        st["positions"] = torch.cat([torch.arange(n, dtype=torch.int32) + (0 if packed else 2 * h + 5)
                                     for n, h in zip(new, have)]).cuda()
        st["freqs"] = _frequencies(case)
        st["amplitude"] = 0.1 * math.log(8.0) + 1.0 if case["scaling"] == "bands" else 1.0
        st["new"], st["have"] = new, have
        room = new if packed else [h + n + 3 for h, n in zip(have, new)]
        slots = sum(room)
        st["starts"], st["slot_starts"] = _starts(new), _starts(room)
        if packed:
            st["token_offsets"] = st["slot_offsets"] = st["lens_in"] = st["lens_out"] = None
        else:
            st["token_offsets"], st["slot_offsets"] = _dev(st["starts"], torch.int64), _dev(st["slot_starts"], torch.int64)
            st["lens_in"] = _dev(have, torch.int32)
            st["lens_out"] = torch.zeros_like(st["lens_in"])
        st["Qr"] = torch.empty((total, Hq, D), dtype=dt, device="cuda")
        st["Kc"], st["Vc"] = (torch.zeros((Hkv, slots, D), dtype=dt, device="cuda") for _ in range(2))
        st["norms"] = torch.zeros((Hkv, slots), device="cuda")
        st["pos"] = torch.zeros((Hkv, slots), dtype=torch.int32, device="cuda")
    elif kind == "prompt":
        new, Hq = _spread(case, "new"), case["Hq"]
        have = _spread(case, "have")
        rows = [h + n for h, n in zip(have, new)]
        st["Q"] = torch.randn((sum(new), Hq, D), generator=gen, device="cuda").to(dt)
        st["K"] = _keys(gen, Hkv, rows, D).to(dt)
        st["V"] = torch.randn((Hkv, sum(rows), D), generator=gen, device="cuda").to(dt)
        st["new"], st["rows"] = new, rows
        st["q_offsets"], st["kv_offsets"] = _dev(_starts(new), torch.int64), _dev(_starts(rows), torch.int64)
        st["O"] = torch.empty((sum(new), Hq, D), dtype=dt, device="cuda")
        if own:
            import paper_2406_11430_amd as l2kv
            ws = l2kv.l2kv_prompt_attn_workspace_bytes(len(new), Hq, Hkv, sum(new), max(rows), D, dt)
            st["workspace"] = torch.zeros(ws, dtype=torch.uint8, device="cuda")
    elif kind == "tree":
        nodes, have, Hq = _spread(case, "nodes"), _spread(case, "have"), case["Hq"]
        room = [h + 16 for h in have]
        st["Q"] = torch.randn((sum(nodes), Hq, D), generator=gen, device="cuda").to(dt)
        st["Kc"] = _keys(gen, Hkv, room, D).to(dt)
        st["Vc"] = torch.randn((Hkv, sum(room), D), generator=gen, device="cuda").to(dt)
        st["Kt"] = _keys(gen, Hkv, nodes, D).to(dt)
        st["Vt"] = torch.randn((Hkv, sum(nodes), D), generator=gen, device="cuda").to(dt)
        st["mask"] = _tree_masks(gen_cpu, nodes, (max(nodes) + 31) // 32).cuda()
        st["nodes"], st["have"], st["slot_starts"] = nodes, have, _starts(room)
        st["node_offsets"], st["slot_offsets"] = _dev(_starts(nodes), torch.int64), _dev(_starts(room), torch.int64)
        st["lens"] = _dev(have, torch.int32)
        st["O"] = torch.empty((sum(nodes), Hq, D), dtype=dt, device="cuda")
        if own:
            import paper_2406_11430_amd as l2kv
            ws = l2kv.l2kv_tree_attn_workspace_bytes(len(nodes), Hq, Hkv, sum(nodes), max(have), D, dt)
            st["workspace"] = torch.zeros(ws, dtype=torch.uint8, device="cuda")
    else:
        nodes, have = _spread(case, "nodes"), _spread(case, "have")
        length = [min(p, n) for p, n in zip(_spread(case, "path"), nodes)]
        planes, longest = case["L"] * Hkv, max(length)
        room = [h + longest for h in have]
        total, slots = sum(nodes), sum(room)
        st["Kt"] = _keys(gen, planes, nodes, D).to(dt)
        st["Vt"] = torch.randn((planes, total, D), generator=gen, device="cuda").to(dt)
        st["norms_t"] = st["Kt"].float().square().sum(-1)
        st["pos_t"] = (torch.arange(total, dtype=torch.int32, device="cuda") + 1000).expand(planes, total).contiguous()
        path = torch.zeros((len(nodes), longest), dtype=torch.int32)
        for s, (n, m) in enumerate(zip(nodes, length)):
            path[s, :m] = torch.randperm(n, generator=gen_cpu)[:m].sort().values.to(torch.int32)
        st["path_host"], st["nodes"], st["have"], st["length"] = path.tolist(), nodes, have, length
        st["slot_starts"] = _starts(room)
        st["path"], st["path_lens"] = path.cuda(), _dev(length, torch.int32)
        st["node_offsets"], st["slot_offsets"] = _dev(_starts(nodes), torch.int64), _dev(st["slot_starts"], torch.int64)
        st["lens_in"] = _dev(have, torch.int32)
        st["lens_out"] = torch.zeros_like(st["lens_in"])
        st["Kc"], st["Vc"] = (torch.zeros((planes, slots, D), dtype=dt, device="cuda") for _ in range(2))
        st["norms"] = torch.zeros((planes, slots), device="cuda")
        st["pos"] = torch.zeros((planes, slots), dtype=torch.int32, device="cuda")
    return st


# ---------------------------------------------------------------------------- one pass
def _cache_outputs(st):
    out = {"Kc": st["Kc"], "Vc": st["Vc"], "norms": st["norms"], "pos": st["pos"]}
    if st["lens_out"] is not None:
        out["lens"] = st["lens_out"]
    return out


def run(st):
    if own:
        return _run_own(st)
    return {"rotary": _plain_rotary, "prompt": _plain_prompt, "tree": _plain_tree, "path": _plain_path}[st["kind"]](st)


def _run_own(st):
    import paper_2406_11430_amd as l2kv
    kind = st["kind"]
    if kind == "rotary":
        l2kv.l2kv_rotary_append(st["Q"], st["K"], st["V"], st["positions"], st["freqs"], st["Qr"], st["Kc"], st["Vc"], st["norms"],
                                st["pos"], st["token_offsets"], st["slot_offsets"], st["lens_in"], st["lens_out"],
                                layout=LAYOUTS[st["case"]["layout"]], amplitude=st["amplitude"])
        return {"Qr": st["Qr"], **_cache_outputs(st)}
    if kind == "prompt":
        l2kv.l2kv_prompt_attn(st["Q"], st["K"], st["V"], st["q_offsets"], st["kv_offsets"], None, max(st["rows"]), st["O"],
                              st["workspace"])
        return st["O"]
    if kind == "tree":
        l2kv.l2kv_tree_attn(st["Q"], st["Kc"], st["Vc"], st["lens"], st["slot_offsets"], max(st["have"]), st["Kt"], st["Vt"],
                            st["node_offsets"], st["mask"], st["O"], st["workspace"])
        return st["O"]
    l2kv.l2kv_stream_append_path(st["Kt"], st["Vt"], st["norms_t"], st["pos_t"], st["node_offsets"], st["path"], st["path_lens"],
                                 st["slot_offsets"], st["lens_in"], st["lens_out"], st["Kc"], st["Vc"], st["norms"], st["pos"])
    return _cache_outputs(st)


def _plain_rotary(st):
    # in 64 bits: the norms are of the rows as stored, so a key that rounds the other way changes its norm
    case = st["case"]
    R, angle = case["rot"], st["positions"].double()[:, None, None] * st["freqs"]
    cos, sin = torch.cos(angle) * st["amplitude"], torch.sin(angle) * st["amplitude"]

    def rotated(x):
        y = x.double()
        if case["layout"] == "half":
            a, b = y[..., :R // 2], y[..., R // 2:R]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = y[..., 0:R:2], y[..., 1:R:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([turned.to(x.dtype), x[..., R:]], -1)

    Qr, K = rotated(st["Q"]), rotated(st["K"])
    norms = K.float().square().sum(-1)
    for s, n in enumerate(st["new"]):
        src, dst = st["starts"][s], st["slot_starts"][s] + st["have"][s]
        st["Kc"][:, dst:dst + n] = K[src:src + n].transpose(0, 1)
        st["Vc"][:, dst:dst + n] = st["V"][src:src + n].transpose(0, 1)
        st["norms"][:, dst:dst + n] = norms[src:src + n].t()
        st["pos"][:, dst:dst + n] = st["positions"][src:src + n]
    if st["lens_out"] is not None:
        ends = torch.tensor([h + n for h, n in zip(st["have"], st["new"])], dtype=torch.int32, device="cuda")
        st["lens_out"].copy_(ends)
    return {"Qr": Qr, **_cache_outputs(st)}


def _softmax_rows(scores, V):
    """Rows of scores (-inf where masked, at least one left) over the values."""
    p = torch.exp(scores - scores.max(-1, keepdim=True).values)
    return (p @ V) / p.sum(-1, keepdim=True)


def _plain_prompt(st):
    case = st["case"]
    G, D = case["Hq"] // case["Hkv"], case["D"]
    scale, out = 1.0 / math.sqrt(D), torch.empty_like(st["O"])
    q0 = k0 = 0
    for n, rows in zip(st["new"], st["rows"]):
        Q = st["Q"][q0:q0 + n].float()
        for h in range(case["Hkv"]):
            K, V = st["K"][h, k0:k0 + rows].float(), st["V"][h, k0:k0 + rows].float()
            step = max(256, (1 << 28) // (rows * G))
            for a in range(0, n, step):
                b = min(n, a + step)
                last = rows - n + b                                           # keys the last of these queries sees
                q = Q[a:b, h * G:(h + 1) * G].transpose(0, 1) * scale         # [G, queries, D]
                scores = q.reshape(-1, D) @ K[:last].t().contiguous()
                limit = torch.arange(a, b, device="cuda")[:, None] + (rows - n)
                hidden = torch.arange(last, device="cuda")[None] > limit
                scores = scores.view(G, b - a, last).masked_fill(hidden, -math.inf).view(-1, last)
                o = _softmax_rows(scores, V[:last])
                out[q0 + a:q0 + b, h * G:(h + 1) * G] = o.view(G, b - a, D).transpose(0, 1).to(out.dtype)
        q0, k0 = q0 + n, k0 + rows
    return out


def _bits(mask, n):
    """[rows, words] int32 -> [rows, n] truth values."""
    j = torch.arange(n, device=mask.device)
    return ((mask[:, j // 32] >> (j % 32).int()) & 1).bool()


def _plain_tree(st):
    case = st["case"]
    G, D, Hkv = case["Hq"] // case["Hkv"], case["D"], case["Hkv"]
    scale, out = 1.0 / math.sqrt(D), torch.empty_like(st["O"])
    t0 = 0
    for n, have, c0 in zip(st["nodes"], st["have"], st["slot_starts"]):
        K = torch.cat([st["Kc"][:, c0:c0 + have], st["Kt"][:, t0:t0 + n]], 1).float()
        V = torch.cat([st["Vc"][:, c0:c0 + have], st["Vt"][:, t0:t0 + n]], 1).float()
        q = st["Q"][t0:t0 + n].float().view(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D) * scale
        scores = torch.bmm(q.contiguous(), K.transpose(1, 2).contiguous()).view(Hkv, G, n, have + n)
        seen = torch.cat([torch.ones((n, have), dtype=torch.bool, device="cuda"), _bits(st["mask"][t0:t0 + n], n)], 1)
        scores = scores.masked_fill(~seen, -math.inf).view(Hkv, G * n, have + n)
        o = _softmax_rows(scores, V)
        out[t0:t0 + n] = o.view(Hkv, G, n, D).permute(2, 0, 1, 3).reshape(n, Hkv * G, D).to(out.dtype)
        t0 += n
    return out


def _plain_path(st):
    t0 = 0
    for s, n in enumerate(st["nodes"]):
        m, dst = st["length"][s], st["slot_starts"][s] + st["have"][s]
        rows = st["path"][s, :m].long() + t0
        for to, src in (("Kc", "Kt"), ("Vc", "Vt"), ("norms", "norms_t"), ("pos", "pos_t")):
            st[to][:, dst:dst + m] = st[src][:, rows]
        t0 += n
    st["lens_out"].copy_(st["lens_in"] + st["path_lens"])
    return _cache_outputs(st)


# ---------------------------------------------------------------------------- what it has to do
def work(case):
    es, D, Hkv, n = (4 if case["dtype"] == "f32" else 2), case["D"], case["Hkv"], case["n_seq"]
    if case["kind"] == "rotary":
        tokens, heads = sum(_spread(case, "new")), case["Hq"] + 2 * Hkv
        turned = tokens * (case["Hq"] + Hkv)
        return {"bytes": 2 * tokens * heads * D * es + tokens * (4 + 8 * Hkv) + 4 * case["rot"],
                "flops": 3 * turned * case["rot"] + 2 * tokens * Hkv * D}
    if case["kind"] == "prompt":
        new, have = _spread(case, "new"), _spread(case, "have")
        pairs = sum(a * h + a * (a + 1) // 2 for a, h in zip(new, have))
        rows = sum(new) + sum(have)
        return {"bytes": 2 * sum(new) * case["Hq"] * D * es + 2 * rows * Hkv * D * es, "flops": 4 * D * case["Hq"] * pairs}
    if case["kind"] == "tree":
        nodes, have = _spread(case, "nodes"), _spread(case, "have")
        # of the nodes, at least each itself
        pairs = sum(a * (h + 1) for a, h in zip(nodes, have))
        return {"bytes": 2 * sum(nodes) * case["Hq"] * D * es + 2 * (sum(nodes) + sum(have)) * Hkv * D * es,
                "flops": 4 * D * case["Hq"] * pairs}
    nodes = _spread(case, "nodes")
    rows = sum(min(p, a) for p, a in zip(_spread(case, "path"), nodes)) * case["L"] * Hkv
    return {"bytes": 2 * rows * (2 * D * es + 8) + 4 * n, "flops": 0}


# ---------------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"rotary": _exact_rotary, "prompt": _exact_prompt, "tree": _exact_tree, "path": _exact_path}[case["kind"]](st, case)


def _exact_rotary(st, case):
    R = case["rot"]
    i = torch.arange(R // 2, device="cuda")
    first, second = (i, i + R // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
    unit = torch.polar(torch.full((len(st["positions"]), R // 2), float(st["amplitude"]), dtype=torch.float64, device="cuda"),
                       torch.outer(st["positions"].double(), st["freqs"]))[:, None]
    turned = []
    for x in (st["Q"], st["K"]):
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * unit
        y[..., first], y[..., second] = z.real, z.imag
        turned.append(y)
    Qr, K = turned
    stored = K.to(DTYPES[case["dtype"]]).double()                 # the norms are of the rows as stored
    Kc, Vc = st["Kc"].double(), st["Vc"].double()
    norms, pos = st["norms"].double(), st["pos"].clone()
    where = torch.cat([torch.arange(n) + b + h for n, h, b in zip(st["new"], st["have"], st["slot_starts"])]).cuda()
    Kc[:, where], Vc[:, where] = K.transpose(0, 1), st["V"].double().transpose(0, 1)
    norms[:, where] = (stored * stored).sum(-1).t()
    pos[:, where] = st["positions"].expand(case["Hkv"], -1)
    out = {"Qr": Qr, "Kc": Kc, "Vc": Vc, "norms": norms, "pos": pos}
    if st["lens_out"] is not None:
        out["lens"] = torch.tensor([h + n for h, n in zip(st["have"], st["new"])], dtype=torch.int32, device="cuda")
    return out


def _exact_rows(q, K, V, seen, scale):
    """q [r, D], K and V [n, D], seen [r, n]: the attention of every row, a block of rows at a time."""
    out = []
    step = max(1, (1 << 27) // K.shape[0])
    for a in range(0, q.shape[0], step):
        logits = (q[a:a + step].double() @ K.double().t()) * scale
        logits = torch.where(seen(a, min(a + step, q.shape[0])), logits, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
        out.append(torch.exp(logits - torch.logsumexp(logits, -1, keepdim=True)) @ V.double())
    return torch.cat(out)


def _exact_prompt(st, case):
    G, out = case["Hq"] // case["Hkv"], torch.empty_like(st["O"], dtype=torch.float64)
    qs, ks = _starts(st["new"]), _starts(st["rows"])
    for s, (n, rows) in enumerate(zip(st["new"], st["rows"])):
        j = torch.arange(rows, device="cuda")
        for hq in range(case["Hq"]):
            K, V = (st[x][hq // G, ks[s]:ks[s + 1]] for x in ("K", "V"))
            out[qs[s]:qs[s + 1], hq] = _exact_rows(st["Q"][qs[s]:qs[s + 1], hq], K, V,
                                                   lambda a, b: j[None] < torch.arange(a, b, device="cuda")[:, None] + (rows - n + 1),
                                                   case["D"] ** -0.5)
    return out


def _exact_tree(st, case):
    G, out = case["Hq"] // case["Hkv"], torch.empty_like(st["O"], dtype=torch.float64)
    ts = _starts(st["nodes"])
    for s, (n, have) in enumerate(zip(st["nodes"], st["have"])):
        t, c = slice(ts[s], ts[s + 1]), slice(st["slot_starts"][s], st["slot_starts"][s] + have)
        words = st["mask"][t].cpu().tolist()
        seen = torch.tensor([[True] * have + [bool((w[j // 32] >> (j % 32)) & 1) for j in range(n)] for w in words], device="cuda")
        for hq in range(case["Hq"]):
            K, V = (torch.cat([st[x + "c"][hq // G, c], st[x + "t"][hq // G, t]]) for x in ("K", "V"))
            out[t, hq] = _exact_rows(st["Q"][t, hq], K, V, lambda a, b: seen[a:b], case["D"] ** -0.5)
    return out


def _exact_path(st, case):
    out = {"Kc": st["Kc"].double(), "Vc": st["Vc"].double(), "norms": st["norms"].double(), "pos": st["pos"].clone()}
    ts = _starts(st["nodes"])
    src = [ts[s] + j for s, row in enumerate(st["path_host"]) for j in row[:st["length"][s]]]
    dst = [b + h + j for b, h, m in zip(st["slot_starts"], st["have"], st["length"]) for j in range(m)]
    for to, frm in (("Kc", "Kt"), ("Vc", "Vt"), ("norms", "norms_t"), ("pos", "pos_t")):
        out[to][:, dst] = st[frm][:, src].to(out[to].dtype)
    out["lens"] = torch.tensor([h + m for h, m in zip(st["have"], st["length"])], dtype=torch.int32, device="cuda")
    return out
