"""What the performance of the key/value cache's operators is measured on: s2o_decode, s2o_key_weights and s2o_evict, in their
plain form (elementary torch operations in 32 bits) and through the framework's entry points.

A case is a dict of plain values:
  op       decode   B sequences attend one shared cache and each its own rows behind it
           weights  what every key of a cache was worth to the queries: softmax weights added up over them
           evict    the cache compacted to the `keep` rows of the largest weights, the first `sink` and the last `recent` among them
  Z B H Hkv D T     caches, sequences of a cache, query heads, key/value heads, head dimension, query tokens of a sequence
  L own             rows of a shared cache and of a sequence's own one
  ragged            1: the caches are filled to different lengths, some of them empty
  dtype             bf16 or f16
  layout            packed ([.., heads, rows, D]) or token ([.., rows, heads, D], described by strides)
  causal given      weights: the queries are the cache's last T tokens; their softmax's normaliser is an input (and so are weights
                    to add to)
  keep sink recent  evict
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}

_BASE = dict(op="decode", Z=1, B=1, H=32, Hkv=8, D=128, T=1, L=0, own=0, ragged=0, dtype="bf16", layout="packed", causal=0, given=0,
             keep=0, sink=0, recent=0)


def _case(name, **kw):
    return dict(_BASE, name=name, **kw)


def listed():
    return [
        # the first tokens behind a short prompt: launches and latency are all of it
        _case("decode_first_tokens", B=2, H=8, Hkv=2, L=96, own=24),
        # one sequence behind the longest prompt that fits its cache here: the long axis has to be split
        _case("decode_single_32k", L=32768, own=256),
        # a batch that samples from one prompt, the Llama-3.1-8B head shape
        _case("decode_32_over_32k", B=32, L=32768, own=512, ragged=1),
        # the longest prompt of the workloads and a large batch
        _case("decode_64_over_128k", B=64, L=131072, own=1024, ragged=1),
        # several new tokens at once (drafts to be checked), token-major caches of odd and different lengths, some empty
        _case("decode_drafts_ragged_f16", Z=3, B=7, H=12, Hkv=4, D=64, T=5, L=5003, own=333, ragged=1, dtype="f16", layout="token"),
        # eviction behind a prefill: the last queries of the prompt judge its keys
        _case("weights_window_128k", op="weights", T=64, L=131072, causal=1),
        # all queries judge (the "accumulated attention" of a whole prompt)
        _case("weights_all_8k", op="weights", T=8192, L=8192, causal=1),
        # a decoding step's queries add to the weights of the shared cache
        _case("weights_decode_32k", op="weights", B=32, L=32768, given=1),
        # few keys, few queries, odd sizes
        _case("weights_small_f16", op="weights", Z=2, B=3, H=12, Hkv=4, D=64, T=3, L=777, ragged=1, dtype="f16", layout="token"),
        # a long prompt's cache cut to an eighth
        _case("evict_128k", op="evict", L=131072, keep=16384, sink=4, recent=1024),
        # caches of a batch at different lengths, to an odd number of rows
        _case("evict_ragged_f16", op="evict", Z=6, Hkv=4, H=4, D=64, L=20001, keep=2777, sink=4, recent=100, ragged=1, dtype="f16", layout="token"),
        # the smallest
        _case("evict_small", op="evict", H=2, Hkv=2, L=300, keep=100, sink=4, recent=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("decode", "weights", "evict")}
    while True:
        c = dict(_BASE)
        c["op"] = rng.choice(["decode", "decode", "weights", "weights", "evict"])
        c["H"], c["Hkv"] = rng.choice([(1, 1), (4, 4), (8, 1), (12, 4), (14, 2), (16, 2), (32, 8), (32, 8), (40, 8)])
        c["Z"] = rng.choice([1, 1, 2, 3, 5])
        c["D"] = rng.choice([64, 128, 128])
        c["dtype"] = rng.choice(["bf16", "bf16", "f16"])
        c["layout"] = rng.choice(["packed", "packed", "token"])
        c["ragged"] = rng.choice([0, 1])
        c["L"] = _log(rng, 16, 131072)
        if c["op"] == "decode":
            c["B"], c["T"], c["own"] = _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 4, 7]), rng.choice([0, _log(rng, 1, 2048), _log(rng, 1, 2048)])
            if rng.random() < 0.1:
                c["L"], c["own"] = 0, max(1, c["own"])
        elif c["op"] == "weights":
            c["causal"] = rng.choice([0, 1])
            if c["causal"]:
                c["T"] = min(c["L"], _log(rng, 1, 8192))
            else:
                c["B"], c["T"], c["given"] = _log(rng, 1, 64), rng.choice([1, 1, 2, 5]), rng.choice([0, 1])
        else:
            c["H"] = c["Hkv"]
            c["keep"] = _log(rng, 1, c["L"])
            c["sink"] = rng.choice([0, min(4, c["keep"])])
            c["recent"] = rng.randint(0, (c["keep"] - c["sink"]) // 2)
        if _cost(c) > most[c["op"]] or c["Z"] * c["Hkv"] * c["L"] > 8 * 131072 or c["Z"] * c["B"] * c["H"] * c["T"] * c["L"] > 32 * 8192 * 8192:
            continue
        return c


# ---------------------------------------------------------------------------------- inputs
def _lens(case):
    """Rows in the shared caches and in the sequences' own ones: a property of the case."""
    Z, B, L, n = case["Z"], case["B"], case["L"], case["own"]
    if not case["ragged"]:
        return [L] * Z, [n] * (Z * B)
    r = random.Random(1000 * L + n)
    shared = [r.randint(L // 2, L) for _ in range(Z)]
    if Z > 2:
        shared[1] = 0
    each = [r.randint(0, n) for _ in range(Z * B)]
    each[-1] = n
    return shared, each


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)


def _stored(x, dtype, layout):
    """Rounded to the cache's type and laid out in memory; the view is [.., heads, rows, D] either way."""
    x = x.to(dtype)
    return x.transpose(-3, -2).contiguous().transpose(-3, -2) if layout == "token" else x.contiguous()


def _strides(x):
    return tuple(x.stride()[:-1])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    Z, B, H, Hkv, D, T, L, n = (case[k] for k in ("Z", "B", "H", "Hkv", "D", "T", "L", "own"))
    dtype, lay = TYPES[case["dtype"]], case["layout"]
    shared, each = _lens(case)
    s = {"c": dict(case), "lens": torch.tensor(shared, dtype=torch.int32, device=DEV) if case["ragged"] else None}
    # keys as a trained head has them: N(0,1), a few heavy ones that every query is drawn to, the first four among them
    u = _randn(gen, Z, Hkv, 1, D)
    u = u / u.norm(dim=-1, keepdim=True)
    if L:
        K = _randn(gen, Z, Hkv, L, D)
        heavy = torch.rand((Z, Hkv, L, 1), generator=gen, device=DEV) < 0.005
        heavy[:, :, :4] = True
        K += heavy * (6.0 * u)
        s["K"] = _stored(K, dtype, lay)
        del K, heavy
        if case["op"] != "weights":
            s["V"] = _stored(_randn(gen, Z, Hkv, L, D), dtype, lay)
    if case["op"] != "evict":
        q = _randn(gen, Z, B, H, T, D) + 3.0 * u.repeat_interleave(H // Hkv, 1)[:, None]
        s["Q"] = _stored(q, dtype, lay)
    if case["op"] == "decode" and n:
        s["own_K"], s["own_V"] = (_stored(_randn(gen, Z, B, Hkv, n, D), dtype, lay) for _ in range(2))
        s["own_lens"] = torch.tensor(each, dtype=torch.int32, device=DEV).view(Z, B) if case["ragged"] else None
    if case["op"] == "weights" and case["given"]:
        # of a softmax over more than these keys: sum of L log-normal terms, and then some
        s["lse"] = math.log(L) + 0.5 + 1.0 * torch.rand((Z, B, H, T), generator=gen, device=DEV)
        s["prev"] = torch.rand((Z, Hkv, L), generator=gen, device=DEV)
    if case["op"] == "evict":
        w = torch.exp(2.0 * _randn(gen, Z, Hkv, L))
        # weights of keys that nobody looked at are zero, and equal ones are common
        s["weights"] = torch.where(torch.rand((Z, Hkv, L), generator=gen, device=DEV) < 0.05, torch.zeros_like(w), torch.round(64.0 * w) / 64.0)
        # the compacted cache is a buffer that the program keeps
        keep = case["keep"]
        shape = (Z, keep, Hkv, D) if lay == "token" else (Z, Hkv, keep, D)
        s["out_K"], s["out_V"] = (torch.zeros(shape, dtype=dtype, device=DEV) for _ in range(2))
        if lay == "token":
            s["out_K"], s["out_V"] = s["out_K"].transpose(1, 2), s["out_V"].transpose(1, 2)
        s["out_weights"] = torch.zeros((Z, Hkv, keep), dtype=torch.float32, device=DEV)
        s["kept"] = torch.zeros((Z, Hkv, keep), dtype=torch.int32, device=DEV)
    if case["op"] == "weights":
        s["out"] = torch.zeros((Z, Hkv, L), dtype=torch.float32, device=DEV)
    if own:
        s["call"] = _kept_by_a_program(s)
    return s


def _kept_by_a_program(s):
    """The description of the call and its workspace, which a program makes once for a shape."""
    import paper_2602_22575_amd as s2o
    c = s["c"]
    dtype, st = TYPES[c["dtype"]], lambda name: _strides(s[name]) if name in s and c["layout"] == "token" else None
    given = lambda **kw: {k: v for k, v in kw.items() if v is not None}  # noqa: E731
    if c["op"] == "decode":
        p = s2o.make_decode_params(c["Z"], c["B"], c["H"], c["Hkv"], c["D"], c["T"], c["L"], c["own"], dtype=dtype, **given(
            q_stride=st("Q"), o_stride=st("Q"), k_stride=st("K"), v_stride=st("V"), own_k_stride=st("own_K"), own_v_stride=st("own_V")))
        size = s2o.s2o_decode_sizes(p)["scratch"]
    elif c["op"] == "weights":
        p = s2o.make_weights_params(c["Z"], c["B"], c["H"], c["Hkv"], c["D"], c["T"], c["L"], dtype=dtype, causal=c["causal"], **given(
            q_stride=st("Q"), k_stride=st("K")))
        size = s2o.s2o_key_weights_sizes(p)["scratch"]
    else:
        p = s2o.make_evict_params(c["Z"], c["Hkv"], c["D"], c["L"], c["keep"], sink=c["sink"], recent=c["recent"], dtype=dtype, **given(
            k_stride=st("K"), v_stride=st("V"), out_k_stride=st("out_K"), out_v_stride=st("out_V")))
        size = s2o.s2o_evict_sizes(p)["scratch"]
    out = {"params": p, "scratch": torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)}
    if c["op"] == "decode":
        out["O"] = torch.empty_like(s["Q"])          # (keeps the layout)
        out["lse"] = torch.empty((c["Z"], c["B"], c["H"], c["T"]), dtype=torch.float32, device=DEV)
    return out


# ---------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return _RUN_OWN[s["c"]["op"]](s)
    return _RUN_PLAIN[s["c"]["op"]](s)


def _own_decode(s):
    import paper_2602_22575_amd as s2o
    k = s["call"]
    O, lse = s2o.s2o_decode(s["Q"], s.get("K"), s.get("V"), k["params"], own_K=s.get("own_K"), own_V=s.get("own_V"), lens=s["lens"],
                            own_lens=s.get("own_lens"), O=k["O"], lse=k["lse"], scratch=k["scratch"])
    return {"O": O, "lse": lse}


def _own_weights(s):
    import paper_2602_22575_amd as s2o
    k = s["call"]
    return {"weights": s2o.s2o_key_weights(s["Q"], s["K"], k["params"], lse=s.get("lse"), lens=s["lens"], prev=s.get("prev"), out=s["out"],
                                           scratch=k["scratch"])}


def _own_evict(s):
    import paper_2602_22575_amd as s2o
    k = s["call"]
    e = s2o.s2o_evict(s["K"], s["V"], s["weights"], k["params"], lens=s["lens"], out_K=s["out_K"], out_V=s["out_V"], out_weights=s["out_weights"],
                      kept=s["kept"], scratch=k["scratch"])
    return {"K": e.K, "V": e.V, "weights": e.weights, "kept": e.kept, "lens": e.lens}


def _grouped(q, Hkv):
    """[Z,B,H,T,D] in 32 bits -> the query rows of a key/value head, [Z,Hkv,B,G,T,D]."""
    Z, B, H, T, D = q.shape
    return q.float().view(Z, B, Hkv, H // Hkv, T, D).transpose(1, 2)


def _filled(rows, lens, Z):
    """[Z, rows] truth values: which rows of the caches hold a token."""
    at = torch.arange(rows, device=DEV)
    return (at[None] < lens[:, None]) if lens is not None else torch.ones((Z, rows), dtype=torch.bool, device=DEV)


def _plain_decode(s):
    c = s["c"]
    Z, B, H, Hkv, D, T, L, n = (c[k] for k in ("Z", "B", "H", "Hkv", "D", "T", "L", "own"))
    G, scale, low = H // Hkv, 1.0 / math.sqrt(D), float("-inf")
    q = _grouped(s["Q"].contiguous(), Hkv).contiguous()
    parts, values = [], []
    if L:
        x = torch.matmul(q.view(Z, Hkv, B * G * T, D), s["K"].float().transpose(-1, -2)) * scale
        x = x.masked_fill(~_filled(L, s["lens"], Z)[:, None, None], low)
        parts.append(x.view(Z, Hkv, B, G * T, L))
    if n:
        x = torch.matmul(q.view(Z, Hkv, B, G * T, D), s["own_K"].float().transpose(1, 2).transpose(-1, -2)) * scale
        lens = s["own_lens"] if s["own_lens"] is not None else torch.full((Z, B), n, device=DEV)
        last = lens[:, None, :, None] - T + torch.arange(T, device=DEV)             # the row that query t ends at
        hidden = torch.arange(n, device=DEV) > last[..., None]                      # [Z,1,B,T,n]
        x = x.view(Z, Hkv, B, G, T, n).masked_fill(hidden[:, :, :, None], low)
        parts.append(x.view(Z, Hkv, B, G * T, n))
    m = torch.stack([x.amax(-1) for x in parts]).amax(0)
    some = m > low
    e = [torch.exp(x - torch.where(some, m, torch.zeros_like(m))[..., None]) for x in parts]
    total = sum(x.sum(-1) for x in e)
    o = 0.0
    if L:
        o = o + torch.matmul(e[0].view(Z, Hkv, B * G * T, L), s["V"].float()).view(Z, Hkv, B, G * T, D)
    if n:
        o = o + torch.matmul(e[-1], s["own_V"].float().transpose(1, 2))
    o = torch.where(some[..., None], o / total[..., None], torch.zeros_like(o))
    lse = torch.where(some, m + torch.log(total), m)
    back = lambda x: x.reshape(Z, Hkv, B, G, T, -1).transpose(1, 2).reshape(Z, B, H, T, -1)  # noqa: E731
    return {"O": back(o).to(s["Q"].dtype), "lse": back(lse).squeeze(-1)}


def _plain_weights(s):
    c = s["c"]
    Z, B, H, Hkv, D, T, L = (c[k] for k in ("Z", "B", "H", "Hkv", "D", "T", "L"))
    G, scale, low = H // Hkv, 1.0 / math.sqrt(D), float("-inf")
    q = _grouped(s["Q"].contiguous(), Hkv).contiguous()
    x = (torch.matmul(q.view(Z, Hkv, B * G * T, D), s["K"].float().transpose(-1, -2)) * scale).view(Z, Hkv, B * G, T, L)
    seen = _filled(L, s["lens"], Z)[:, None]                                         # [Z,1,L]
    if c["causal"]:
        lens = s["lens"] if s["lens"] is not None else torch.full((Z,), L, device=DEV)
        last = lens[:, None] - T + torch.arange(T, device=DEV)
        seen = seen & (torch.arange(L, device=DEV) <= last[..., None])               # [Z,T,L]
    x = x.masked_fill(~seen[:, None, None], low)
    if "lse" in s:
        p = torch.exp(x - s["lse"].view(Z, B, Hkv, G, T).transpose(1, 2).reshape(Z, Hkv, B * G, T, 1))
    else:
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - torch.where(m > low, m, torch.zeros_like(m)))
        p = p / torch.where(m > low, p.sum(-1, keepdim=True), torch.ones_like(m))
    w = p.sum((2, 3))
    if "prev" in s:
        w = w + s["prev"]
    return {"weights": torch.where(_filled(L, s["lens"], Z)[:, None], w, s["out"])}


def _plain_evict(s):
    c = s["c"]
    Z, Hkv, D, L, keep, sink, recent = (c[k] for k in ("Z", "Hkv", "D", "L", "keep", "sink", "recent"))
    n = s["lens"].long() if s["lens"] is not None else torch.full((Z,), L, device=DEV)
    at = torch.arange(L, device=DEV)
    rank = s["weights"].clone()
    rank = torch.where(((at < sink) | (at >= n[:, None] - recent))[:, None], torch.full_like(rank, float("inf")), rank)
    rank = torch.where((at < n[:, None])[:, None], rank, torch.full_like(rank, float("-inf")))
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    m = torch.clamp(n, max=keep)
    slot = torch.arange(keep, device=DEV)
    valid = (slot < m[:, None])[:, None].expand(Z, Hkv, keep)
    best = torch.sort(torch.where(valid, best, torch.full_like(best, L)), dim=-1).values
    row = torch.where(valid, best, torch.zeros_like(best))
    take = lambda x, out: torch.where(valid[..., None], torch.gather(x, 2, row[..., None].expand(Z, Hkv, keep, D)), out)  # noqa: E731
    return {"K": take(s["K"], s["out_K"]), "V": take(s["V"], s["out_V"]),
            "weights": torch.where(valid, torch.gather(s["weights"], 2, row), s["out_weights"]),
            "kept": torch.where(valid, best.int(), s["kept"]), "lens": m.int()}


_RUN_PLAIN = {"decode": _plain_decode, "weights": _plain_weights, "evict": _plain_evict}
_RUN_OWN = {"decode": _own_decode, "weights": _own_weights, "evict": _own_evict}


# ---------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    Z, B, H, Hkv, D, T, L = (c[k] for k in ("Z", "B", "H", "Hkv", "D", "T", "L"))
    shared, each = _lens(c)
    n, G = sum(shared), H // Hkv
    if c["op"] == "decode":
        rows = Z * B * H * T
        nbytes = rows * (2 * 2 * D + 4) + 2 * 2 * D * Hkv * (n + (sum(each) if c["own"] else 0))
        pairs = B * n * H * T
        if c["own"]:
            pairs += H * sum(max(0, p - T + t + 1) for p in each for t in range(T))
        return {"bytes": nbytes, "flops": 4 * D * pairs}
    if c["op"] == "weights":
        nbytes = 2 * D * Z * B * H * T + Hkv * n * (2 * D + 4)
        if c["given"]:
            nbytes += 4 * Z * B * H * T + 4 * Hkv * n
        if c["causal"]:
            pairs = 0
            for m in shared:
                first = max(0, T - m)                # queries in front of it see nothing
                count = T - first
                pairs += B * H * (count * (m - T + first + 1) + count * (count - 1) // 2)
        else:
            pairs = B * H * T * n
        return {"bytes": nbytes, "flops": (2 if c["given"] else 4) * D * pairs}
    kept = sum(min(m, c["keep"]) for m in shared)
    return {"bytes": Hkv * (4 * n + kept * (2 * 2 * 2 * D + 2 * 4)), "flops": 0}


def _cost(c):
    w = work(c)
    return w["flops"] / 1e12 + w["bytes"] / 4e9


# ---------------------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    Z, B, H, Hkv, D, T, L, n = (case[k] for k in ("Z", "B", "H", "Hkv", "D", "T", "L", "own"))
    G = H // Hkv
    shared, each = _lens(case)
    scale = 1.0 / math.sqrt(D)
    if case["op"] == "decode":
        O = torch.zeros((Z, B, H, T, D), dtype=torch.float64, device=DEV)
        lse = torch.full((Z, B, H, T), float("-inf"), dtype=torch.float64, device=DEV)
        for z in range(Z):
            for g in range(Hkv):
                heads = slice(g * G, (g + 1) * G)
                q = s["Q"][z, :, heads].double() * scale                             # [B,G,T,D]
                k0, v0 = (s[x][z, g, :shared[z]].double() if L else torch.zeros((0, D), dtype=torch.float64, device=DEV) for x in "KV")
                for b in range(B):
                    p = each[z * B + b] if n else 0
                    k1, v1 = (s[x][z, b, g, :p].double() if n else k0[:0] for x in ("own_K", "own_V"))
                    k, v = (torch.cat(x) for x in ((k0, k1), (v0, v1))) if p else (k0, v0)
                    for t in range(T):
                        see = shared[z] + max(0, p - T + t + 1) if n else shared[z]
                        if see:
                            x = q[b, :, t] @ k[:see].T
                            a = torch.logsumexp(x, -1, keepdim=True)
                            O[z, b, heads, t] = torch.exp(x - a) @ v[:see]
                            lse[z, b, heads, t] = a[:, 0]
        return {"O": O, "lse": lse}
    if case["op"] == "evict":
        out = {k: s[x].double() for k, x in (("K", "out_K"), ("V", "out_V"), ("weights", "out_weights"))}
        for z in range(Z):
            m = shared[z]
            for g in range(Hkv):
                w = s["weights"][z, g, :m].double().cpu().numpy()
                free = np.arange(case["sink"], max(case["sink"], m - case["recent"]))
                best = free[np.lexsort((free, -w[free]))]
                there = np.setdiff1d(np.arange(m), free)
                at = np.sort(np.concatenate([there, best[:max(0, min(m, case["keep"]) - len(there))]]))
                at = torch.from_numpy(at).to(DEV)
                for k, x in (("K", s["K"]), ("V", s["V"]), ("weights", s["weights"])):
                    out[k][z, g, :len(at)] = x[z, g, at].double()
        return dict(out, kept=None, lens=None)
    w = s["out"].double()
    for z in range(Z):
        m = shared[z]
        for g in range(Hkv):
            k = s["K"][z, g, :m].double()
            total = torch.zeros(m, dtype=torch.float64, device=DEV)
            for h in range(g * G, (g + 1) * G):
                for b in range(B):
                    x = (s["Q"][z, b, h].double() @ k.T) * scale                     # [T,m]
                    if case["causal"]:
                        x = x + torch.triu(torch.full((T, m), float("-inf"), dtype=torch.float64, device=DEV), diagonal=m - T + 1)
                    a = s["lse"][z, b, h, :, None].double() if case["given"] else torch.logsumexp(x, -1, keepdim=True)
                    total += torch.where(a > float("-inf"), torch.exp(x - a), torch.zeros_like(x)).sum(0)
            w[z, g, :m] = total + (s["prev"][z, g, :m].double() if case["given"] else 0.0)
    return {"weights": w}
