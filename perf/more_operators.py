"""What is measured of the operators around the cache: norm, position rotation and KV write in one pass; decode attention of
a batch whose requests share prefixes; decode and prefill attention with capped scores, distance bias, window and prefix mask.

``run`` does one pass: in plain torch operations, or (``own``) through this repository's public calls.
"""
import math
import zlib

import numpy as np
import torch

own = False

BS = 16                      # tokens of a block
DEV = "cuda"
EPS = 1e-6                   # of the norms


# ------------------------------------------------------------------------------------------ cases

def listed():
    """Head layouts are those of this repository's configurations (32q/8kv, 28q/4kv at head_dim 128, 4q/2kv and 16q/2kv at 64)."""
    return [
        # a decode step of the small layout: rows of one fused projection, rotation of all channels, no norms
        {"name": "rope-31-4q2kv-d64", "op": "rope", "T": 31, "run": 1, "Hq": 4, "Hk": 2, "D": 64, "rot": 64, "axes": 1, "inter": False, "norm": False, "far": 8000},
        # a decode step of 256 requests, normed queries and keys, far positions
        {"name": "rope-256-32q8kv-d128", "op": "rope", "T": 256, "run": 1, "Hq": 32, "Hk": 8, "D": 128, "rot": 128, "axes": 1, "inter": False, "norm": True, "far": 900000},
        # a prompt chunk with image tokens: three position axes, adjacent channels paired, half of the channels rotated
        {"name": "rope-2049-28q4kv-3axes", "op": "rope", "T": 2049, "run": 683, "Hq": 28, "Hk": 4, "D": 128, "rot": 64, "axes": 3, "inter": True, "norm": True, "far": 4000},
        # a long prompt chunk
        {"name": "rope-16384-32q8kv-d128", "op": "rope", "T": 16384, "run": 1021, "Hq": 32, "Hk": 8, "D": 128, "rot": 128, "axes": 1, "inter": False, "norm": True, "far": 100000},
        # four samples of one short prompt: latency
        {"name": "shared-4over512-4q2kv-d64", "op": "shared", "G": 1, "nlo": 4, "nhi": 4, "plo": 512, "phi": 512, "slo": 1, "shi": 40, "Hq": 4, "Hk": 2, "D": 64},
        # requests of several applications, each with a system prompt of its own, groups of seven heads
        {"name": "shared-9groups-28q4kv", "op": "shared", "G": 9, "nlo": 1, "nhi": 23, "plo": 300, "phi": 6000, "slo": 1, "shi": 900, "Hq": 28, "Hk": 4, "D": 128},
        # one long document, many questions
        {"name": "shared-256over16384-32q8kv", "op": "shared", "G": 1, "nlo": 256, "nhi": 256, "plo": 16384, "phi": 16384, "slo": 17, "shi": 700, "Hq": 32, "Hk": 8, "D": 128},
        # few short sequences, capped scores: latency
        {"name": "sdecode-5x1000-cap-d64", "op": "sdecode", "R": 5, "clo": 1, "chi": 1, "plo": 0, "phi": 999, "Hq": 4, "Hk": 2, "D": 64, "cap": 30.0, "window": 0, "bias": False, "pre": 0},
        # a windowed, capped layer of a decode step over long sequences; the first 16 tokens always seen
        {"name": "sdecode-64x16000-window-cap", "op": "sdecode", "R": 64, "clo": 1, "chi": 1, "plo": 2000, "phi": 16000, "Hq": 32, "Hk": 8, "D": 128, "cap": 50.0, "window": 4096, "bias": False, "pre": 16},
        # prompts with an image part that sees itself whole, window on the rest
        {"name": "sprefill-7x700-prefix-d64", "op": "sprefill", "R": 7, "clo": 5, "chi": 700, "plo": 0, "phi": 0, "Hq": 16, "Hk": 2, "D": 64, "cap": 0.0, "window": 257, "bias": False, "pre": 100},
        # ragged fresh prompts, distance bias, groups of seven
        {"name": "sprefill-24x1500-bias-28q4kv", "op": "sprefill", "R": 24, "clo": 17, "chi": 1500, "plo": 0, "phi": 0, "Hq": 28, "Hk": 4, "D": 128, "cap": 0.0, "window": 0, "bias": True, "pre": 0},
        # one chunk of a long prompt over its cached prefix, capped scores
        {"name": "sprefill-2048over14001-cap", "op": "sprefill", "R": 1, "clo": 2048, "chi": 2048, "plo": 14001, "phi": 14001, "Hq": 32, "Hk": 8, "D": 128, "cap": 50.0, "window": 0, "bias": False, "pre": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "shared", "sdecode", "sprefill"])
    Hq, Hk, D = rng.choice([(32, 8, 128), (64, 8, 128), (4, 2, 64), (28, 4, 128), (8, 8, 64), (6, 2, 128), (16, 2, 64), (5, 1, 64)])
    heads = {"Hq": Hq, "Hk": Hk, "D": D}
    if op == "rope":
        axes = rng.choice([1, 1, 2, 3, 4])
        rot = rng.choice([D, D, D // 2, 2 * rng.randint(axes, D // 2)])
        t = _log_int(rng, 1, min(16384, 16384 * 48 * 128 // ((Hq + 2 * Hk) * D)))
        return {"op": op, "T": t, "run": rng.choice([1, _log_int(rng, 2, 2000)]), **heads, "rot": rot, "axes": axes,
                "inter": rng.random() < 0.5, "norm": rng.random() < 0.7, "far": _log_int(rng, 100, 1000000)}
    if op == "shared":
        g = _log_int(rng, 1, 32)
        nhi = _log_int(rng, 1, max(1, 300 // g))
        # no more scores, and no more bytes of own keys, than the largest listed case has
        phi = max(16, min(_log_int(rng, 16, 20000), (1 << 27) // (g * nhi * Hq), (1 << 27) // (g * Hk * D)))
        shi = max(1, min(_log_int(rng, 1, 4000), (1 << 27) // (g * nhi * Hk * D)))
        return {"op": op, "G": g, "nlo": rng.randint(1, nhi), "nhi": nhi, "plo": rng.choice([0, phi // 2, phi]), "phi": phi,
                "slo": rng.randint(1, shi), "shi": shi, **heads}
    kind = rng.choice(["cap", "window", "bias", "pre", "all"])
    mods = {"cap": rng.choice([5.0, 30.0, 50.0]) if kind in ("cap", "all") or rng.random() < 0.3 else 0.0,
            "window": _log_int(rng, 1, 6000) if kind in ("window", "all") or rng.random() < 0.3 else 0,
            "bias": kind in ("bias", "all"), "pre": _log_int(rng, 1, 500) if kind in ("pre", "all") else 0}
    if op == "sdecode":
        r = _log_int(rng, 1, 200)
        phi = max(1, min(_log_int(rng, 16, 60000), (1 << 28) // (r * Hk * D)))
        return {"op": op, "R": r, "clo": 1, "chi": 1, "plo": rng.randint(0, phi), "phi": phi, **heads, **mods}
    r = _log_int(rng, 1, 32)
    chi = max(1, min(_log_int(rng, 1, 2048), math.isqrt((1 << 29) // (r * Hq))))
    phi = min(rng.choice([0, _log_int(rng, 1, 14000)]), (1 << 29) // (r * chi * Hq))
    return {"op": op, "R": r, "clo": rng.randint(1, chi), "chi": chi, "plo": phi // 2, "phi": phi, **heads, **mods}


def _lengths(case, stream, n, lo, hi):
    """Lengths belong to the case, so that every seed's outputs have the same shapes."""
    text = repr(sorted((k, v) for k, v in case.items() if k != "name"))
    return np.random.RandomState((zlib.crc32(text.encode()) + stream) % (1 << 32)).randint(lo, hi + 1, size=n).astype(np.int64)


def _blocks(L):
    return (L + BS - 1) // BS


def _requests(case):
    """(new tokens, tokens before them) of each request; one new token for a decode step."""
    if case["op"] == "rope":
        n = -(-case["T"] // case["run"])
        new = np.full(n, case["run"], np.int64)
        new[-1] = case["T"] - case["run"] * (n - 1)
        return new, _lengths(case, 3, n, 0, 40)
    if case["op"] == "shared":
        n, p = _groups(case)
        return np.ones(int(n.sum()), np.int64), np.repeat(p, n) + _lengths(case, 4, int(n.sum()), case["slo"], case["shi"]) - 1
    return _lengths(case, 5, case["R"], case["clo"], case["chi"]), _lengths(case, 6, case["R"], case["plo"], case["phi"])


def _groups(case):
    """(requests, shared tokens) of each group; whole blocks are shared."""
    return _lengths(case, 1, case["G"], case["nlo"], case["nhi"]), _lengths(case, 2, case["G"], case["plo"], case["phi"]) // BS * BS


def _seen(case, r_new, r_past):
    """Keys that each of a request's rows sees (a count for every row)."""
    p = r_past + np.arange(r_new)
    first = np.maximum(0, p - case["window"] + 1) if case["window"] else np.zeros_like(p)
    pre = min(case["pre"], r_past + r_new)
    return p - first + 1 + np.minimum(first, pre) + np.maximum(0, pre - 1 - p)


def _touched(case, r_new, r_past):
    """Keys that any of a request's rows sees."""
    first = max(0, r_past - case["window"] + 1) if case["window"] else 0
    pre, total = min(case["pre"], r_past + r_new), r_past + r_new
    return total - first + min(first, pre)


def work(case):
    op, Hq, Hk, D = case["op"], case["Hq"], case["Hk"], case["D"]
    new, past = _requests(case)
    T = int(new.sum())
    if op == "rope":
        # rows in, rotated queries and the cache's rows out; slots and positions
        return {"bytes": T * (2 * 2 * (Hq + 2 * Hk) * D + 8 + 4 * case["axes"]), "flops": 0}
    token = 2 * 2 * Hk * D
    if op == "shared":
        n, p = _groups(case)
        keys = int(p.sum() + (past + 1 - np.repeat(p, n)).sum())
        return {"bytes": keys * token + 2 * T * Hq * D * 2, "flops": 4 * Hq * D * float((past + 1).sum())}
    seen = sum(float(_seen(case, int(c), int(p)).sum()) for c, p in zip(new, past))
    keys = sum(_touched(case, int(c), int(p)) for c, p in zip(new, past))
    return {"bytes": keys * token + 2 * T * Hq * D * 2, "flops": 4 * Hq * D * seen}


# ------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _assign(case, seed):
    """Block tables over a shuffled pool: (int32 [R, width] on the host with -1 behind a request's last block, blocks in all)."""
    new, past = _requests(case)
    need = _blocks(new + past)
    shared = np.zeros_like(need)
    if case["op"] == "shared":
        n, p = _groups(case)
        shared, own_group = np.repeat(p // BS, n), np.repeat(np.arange(len(n)), n)
        start = np.cumsum(p // BS) - p // BS
        at0 = int((p // BS).sum())
    else:
        at0 = 0
    total = at0 + int((need - shared).sum()) + 7
    ids = np.random.RandomState((seed * 31 + 5) % (1 << 31)).permutation(total).astype(np.int32)
    tables = np.full((len(need), int(need.max())), -1, np.int32)
    at = at0
    for r in range(len(need)):
        if shared[r]:
            tables[r, :shared[r]] = ids[start[own_group[r]]:start[own_group[r]] + shared[r]]
        tables[r, shared[r]:need[r]] = ids[at:at + need[r] - shared[r]]
        at += int(need[r] - shared[r])
    return tables, total


def _cache(nb, Hk, D, seed):
    """A filled cache [nb, 2, Hk, BS, D]."""
    g = _generator(seed)
    cache = torch.empty((nb, 2, Hk, BS, D), dtype=torch.bfloat16, device=DEV)
    step = max(1, (1 << 28) // (2 * Hk * BS * D))
    for i in range(0, nb, step):
        n = min(step, nb - i)
        cache[i:i + n] = torch.randn((n, 2, Hk, BS, D), generator=g, device=DEV).to(torch.bfloat16)
    return cache


def _to(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def _slopes(Hq):
    """Slopes of the distance bias: a geometric series over the heads."""
    return (2.0 ** (-8.0 * (torch.arange(Hq, dtype=torch.float64) + 1) / Hq)).to(torch.float32)


def _axis_of_pair(case):
    """Which position each pair of channels turns by: the axes take sections of the pairs, the first one the largest."""
    pairs, axes = case["rot"] // 2, case["axes"]
    cut = [pairs * (i + 1) // (axes + 1) for i in range(axes - 1)]
    return [axes - 1 - sum(i < c for c in cut) for i in range(pairs)]


def _rope_inputs(case, seed):
    """Host and device inputs of the rotation, on the device: projection rows, positions, frequencies, weights, slots."""
    g = _generator(seed + 1)
    T, Hq, Hk, D = case["T"], case["Hq"], case["Hk"], case["D"]
    new, past = _requests(case)
    tables, blocks = _assign(case, seed)
    req = np.repeat(np.arange(len(new)), new)
    pos = np.arange(T) - np.repeat(np.cumsum(new) - new, new) + past[req]
    slots = tables[req, pos // BS].astype(np.int64) * BS + pos % BS
    far = np.random.RandomState((seed * 13 + 1) % (1 << 31)).randint(0, case["far"] + 1, size=len(new))[req]
    positions = np.stack([far + pos] + [(far + pos // (7 * a)) % 5000 for a in range(1, case["axes"])])
    pairs = case["rot"] // 2
    x = {"qkv": torch.randn((T, (Hq + 2 * Hk) * D), generator=g, device=DEV).to(torch.bfloat16),
         "positions": _to(positions if case["axes"] > 1 else positions[0], torch.int32), "slots": _to(slots, torch.int64),
         "inv_freq": (500000.0 ** (-torch.arange(pairs, dtype=torch.float64, device=DEV) / pairs)).to(torch.float32),
         "q_weight": None, "k_weight": None, "blocks": blocks}
    if case["norm"]:
        x["q_weight"] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16)
        x["k_weight"] = (1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16)
    return x


def _split(x, case):
    """Queries, keys and values as views of the projection's rows."""
    T, Hq, Hk, D = case["T"], case["Hq"], case["Hk"], case["D"]
    r = x.view(T, Hq + 2 * Hk, D)
    return r[:, :Hq], r[:, Hq:Hq + Hk], r[:, Hq + Hk:]


def _hold(st, cache, Hq):
    """Puts the cache where the pass finds it: a tensor, or a pool of this repository."""
    if own:
        import paper_2608_23658_b200 as ekv
        nb, _, Hk, _, D = cache.shape
        st["pool"] = ekv.Pool(num_q_heads=Hq, num_kv_heads=Hk, head_dim=D, base_blocks=nb)
        st["cache"] = st["pool"].layer_tensor(0, 0, nb)
        st["cache"].copy_(cache)
    else:
        st["cache"] = cache


def prepare(case, seed):
    op, Hq, Hk, D = case["op"], case["Hq"], case["Hk"], case["D"]
    st = {"op": op, "case": case}
    if op == "rope":
        st.update(_rope_inputs(case, seed))
        _hold(st, _cache(st["blocks"], Hk, D, seed), Hq)
        st["axes"] = _axis_of_pair(case) if case["axes"] > 1 else None
        st["q_out"] = torch.empty((case["T"], Hq, D), dtype=torch.bfloat16, device=DEV)
        return st
    new, past = _requests(case)
    tables, blocks = _assign(case, seed)
    _hold(st, _cache(blocks, Hk, D, seed), Hq)
    T = int(new.sum())
    st.update(tables=_to(tables, torch.int32), lens=_to(new + past, torch.int32), scale=1 / math.sqrt(D), q=_queries(case, T, seed),
              out=torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV))
    if op == "shared":
        n, p = _groups(case)
        st["starts"] = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32))
        st["shared"] = torch.from_numpy(p.astype(np.int32))
        return st
    st.update(cap=case["cap"], window=case["window"], slopes=_slopes(Hq).to(DEV) if case["bias"] else None,
              prefix=torch.full((case["R"],), case["pre"], dtype=torch.int32, device=DEV) if case["pre"] else None)
    st["cu_host"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32))
    st["cu"] = st["cu_host"].to(DEV)
    st["rows"] = int(new.max())
    return st


def _queries(case, T, seed):
    # scores of capped layers reach well into the cap's bend
    mag = 4.0 if case.get("cap") else 1.0
    return (torch.randn((T, case["Hq"], case["D"]), generator=_generator(seed + 1), device=DEV) * mag).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------ one pass

def run(st):
    if own:
        return _run_own(st)
    return {"rope": _plain_rope, "shared": _plain_shared, "sdecode": _plain_scored, "sprefill": _plain_scored}[st["op"]](st)


def _run_own(st):
    pool, op = st["pool"], st["op"]
    if op == "rope":
        q, k, v = _split(st["qkv"], st["case"])
        pool.rope_write_kv(0, q, k, v, st["positions"], st["inv_freq"], st["slots"], q_weight=st["q_weight"], k_weight=st["k_weight"],
                           eps=EPS, interleaved=st["case"]["inter"], axes=st["axes"], q_out=st["q_out"])
        return [st["q_out"], st["cache"]]
    if op == "shared":
        return pool.attn_decode_shared(0, st["q"], st["tables"], st["lens"], st["starts"], st["shared"], st["scale"], out=st["out"])
    if op == "sdecode":
        return pool.attn_decode_scored(0, st["q"], st["tables"], st["lens"], st["scale"], cap=st["cap"], window=st["window"],
                                       slopes=st["slopes"], prefix_lens=st["prefix"], out=st["out"])
    return pool.attn_prefill_chunk_scored(0, st["q"], st["tables"], st["cu"], st["cu_host"], st["lens"], st["scale"], cap=st["cap"],
                                          window=st["window"], slopes=st["slopes"], prefix_lens=st["prefix"], out=st["out"])


def _plain_rope(st):
    case = st["case"]
    pairs, inter = case["rot"] // 2, case["inter"]
    pos = st["positions"].view(case["axes"], -1)
    if st["axes"] is not None:
        pos = pos[torch.tensor(st["axes"], device=DEV)].T                      # [T, pairs]
    else:
        pos = pos[0][:, None]
    angle = pos.double() * st["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turn(x, weight):
        x = x.float()
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
        r, rest = x[..., :2 * pairs], x[..., 2 * pairs:]
        a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :pairs], r[..., pairs:])
        c, d = a * cos - b * sin, b * cos + a * sin
        r = torch.stack([c, d], -1).flatten(-2) if inter else torch.cat([c, d], -1)
        return torch.cat([r, rest], -1).to(torch.bfloat16)

    q, k, v = _split(st["qkv"], case)
    st["q_out"].copy_(turn(q, st["q_weight"]))
    blk, off = st["slots"] // BS, st["slots"] % BS
    st["cache"][blk, 0, :, off] = turn(k, st["k_weight"])
    st["cache"][blk, 1, :, off] = v
    return [st["q_out"], st["cache"]]


def _gathered(st, tables, lens):
    """K and V of tables' rows as float32 [n, Hk, L, D], zero where there is no key."""
    t = tables.long()
    x = st["cache"][t.clamp(min=0)].float()                                    # [n, nb, 2, Hk, BS, D]
    n, nb, _, Hk, _, D = x.shape
    live = (t >= 0)[:, :, None] & (torch.arange(nb * BS, device=DEV).view(nb, BS) < lens.long()[:, None, None])
    x = torch.where(live[:, :, None, None, :, None], x, torch.zeros((), device=DEV))
    x = x.permute(2, 0, 3, 1, 4, 5).reshape(2, n, Hk, nb * BS, D)
    return x[0], x[1]


def _softmax_rows(s, seen):
    s = torch.where(seen, s, torch.full((), -math.inf, device=DEV))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    l = p.sum(-1, keepdim=True)
    return p / torch.where(l > 0, l, torch.ones_like(l))


def _plain_shared(st):
    """A group's shared keys meet all its rows in one product; each request's own keys only its own."""
    q, tables, lens = st["q"].float(), st["tables"], st["lens"]
    _, Hq, D = q.shape
    Hk = st["cache"].shape[2]
    for g, p in enumerate(st["shared"].tolist()):
        a, b = st["starts"][g].item(), st["starts"][g + 1].item()
        n, grp = b - a, Hq // Hk
        if n == 0:
            continue
        x = q[a:b].view(n, Hk, grp, D)
        K, V = _gathered(st, tables[a:b, p // BS:], lens[a:b] - p)
        s = torch.matmul(x, K.transpose(2, 3)) * st["scale"]                   # [n, Hk, grp, own keys]
        seen = (torch.arange(K.shape[2], device=DEV) < (lens[a:b] - p).long()[:, None])[:, None, None]
        rows = x.permute(1, 0, 2, 3).reshape(Hk, n * grp, D)
        Kp, Vp = _gathered(st, tables[a:a + 1, :p // BS], torch.full((1,), p, device=DEV))
        sp = (torch.matmul(rows, Kp[0].transpose(1, 2)) * st["scale"]).view(Hk, n, grp, p).transpose(0, 1)
        w = _softmax_rows(torch.cat([sp, s], -1), torch.cat([torch.ones((1, 1, 1, p), dtype=torch.bool, device=DEV).expand(n, 1, 1, p), seen], -1))
        o = torch.matmul(w[..., p:], V)
        o += torch.matmul(w[..., :p].transpose(0, 1).reshape(Hk, n * grp, p), Vp[0]).view(Hk, n, grp, D).transpose(0, 1)
        st["out"][a:b] = o.reshape(n, Hq, D).to(torch.bfloat16)
    return st["out"]


def _plain_scored(st):
    T, Hq, D = st["q"].shape
    cu, lens = st["cu"].long(), st["lens"].long()
    K, V = _gathered(st, st["tables"], st["lens"])
    R, Hk, Lmax, _ = K.shape
    grp, rows = Hq // Hk, st["rows"]
    c = cu[1:] - cu[:-1]
    i = torch.arange(rows, device=DEV)
    there = i < c[:, None]                                              # [R, rows]
    q = st["q"][(cu[:-1, None] + i).clamp(max=T - 1)].float()           # [R, rows, Hq, D]
    q = q.view(R, rows, Hk, grp, D).permute(0, 2, 3, 1, 4).reshape(R, Hk, grp * rows, D)
    s = (torch.matmul(q, K.transpose(2, 3)) * st["scale"]).view(R, Hk, grp, rows, Lmax)
    if st["cap"]:
        s = st["cap"] * torch.tanh(s / st["cap"])
    p = ((lens - c)[:, None] + i)[..., None]                            # a row's position
    j = torch.arange(Lmax, device=DEV)
    if st["slopes"] is not None:
        s = s - st["slopes"].view(1, Hk, grp, 1, 1) * (p - j).abs().float()[:, None, None]
    seen = j <= p
    if st["window"]:
        seen = seen & (j > p - st["window"])
    if st["prefix"] is not None:
        seen = seen | (j < st["prefix"].long()[:, None, None])
    seen = seen & (j < lens[:, None, None])
    w = _softmax_rows(s, seen[:, None, None]).view(R, Hk, grp * rows, Lmax)
    o = torch.matmul(w, V).view(R, Hk, grp, rows, D).permute(0, 3, 1, 2, 4).reshape(R, rows, Hq, D)
    out = torch.zeros((T + 1, Hq, D), dtype=torch.bfloat16, device=DEV)  # rows that a request does not have go to the last one
    out[torch.where(there, cu[:-1, None] + i, torch.full_like(there, T, dtype=torch.int64))] = o.to(torch.bfloat16)
    return out[:T]


# ------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    op, Hq, Hk, D = case["op"], case["Hq"], case["Hk"], case["D"]
    if op == "rope":
        x = _rope_inputs(case, seed)
        cache = _cache(x["blocks"], Hk, D, seed).double()
        rows, pairs = x["qkv"].double().view(case["T"], Hq + 2 * Hk, D), case["rot"] // 2
        pos = x["positions"].view(case["axes"], -1).double()
        first = list(range(0, 2 * pairs, 2)) if case["inter"] else list(range(pairs))
        axis = _axis_of_pair(case) if case["axes"] > 1 else [0] * pairs
        done = rows.clone()
        if case["norm"]:
            for a, b, w in ((0, Hq, x["q_weight"]), (Hq, Hq + Hk, x["k_weight"])):
                done[:, a:b] = rows[:, a:b] / torch.sqrt(rows[:, a:b].pow(2).sum(-1, keepdim=True) / D + EPS) * w.double()
        heads = slice(0, Hq + Hk)
        for i, f in enumerate(x["inv_freq"].double().tolist()):
            a, b = first[i], first[i] + (1 if case["inter"] else pairs)
            turn = pos[axis[i]][:, None] * f
            u, w = done[:, heads, a].clone(), done[:, heads, b].clone()
            done[:, heads, a] = u * turn.cos() - w * turn.sin()
            done[:, heads, b] = u * turn.sin() + w * turn.cos()
        blk, off = x["slots"] // BS, x["slots"] % BS
        cache[blk, 0, :, off] = done[:, Hq:Hq + Hk]
        cache[blk, 1, :, off] = done[:, Hq + Hk:]
        return [done[:, :Hq].contiguous(), cache]
    new, past = _requests(case)
    tables, blocks = _assign(case, seed)
    cache, T = _cache(blocks, Hk, D, seed), int(new.sum())
    q = _queries(case, T, seed).double()
    slopes = _slopes(Hq).double().to(DEV)
    out, at, grp = torch.empty((T, Hq, D), dtype=torch.float64, device=DEV), 0, Hq // Hk
    for r in range(len(new)):
        c, L = int(new[r]), int(new[r] + past[r])
        kv = cache[_to(tables[r, :_blocks(L)], torch.int64)].double().permute(1, 2, 0, 3, 4).reshape(2, Hk, -1, D)[:, :, :L]
        p, j = torch.arange(L - c, L, device=DEV)[:, None], torch.arange(L, device=DEV)
        seen = p >= j
        if case.get("window"):
            seen = seen & (p - j < case["window"])
        if case.get("pre"):
            seen = seen | (j < case["pre"])
        for h in range(Hk):
            mine = slice(h * grp, (h + 1) * grp)
            s = torch.einsum("chd,ld->hcl", q[at:at + c, mine], kv[0, h]) / math.sqrt(D)
            if case.get("cap"):
                s = case["cap"] * torch.tanh(s / case["cap"])
            if case.get("bias"):
                s = s - slopes[mine, None, None] * (p - j).abs()
            s.masked_fill_(~seen, -math.inf)
            out[at:at + c, mine] = torch.einsum("hcl,ld->chd", torch.softmax(s, -1), kv[1, h])
        at += c
    return out
