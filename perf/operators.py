"""The cases that the calls on an 8-bit KV cache are measured on.

A decoding program that keeps the target's cache in 8 bits makes four kinds of
call: it appends new keys and values (a prompt's, or those of the path that a
verification accepted), it reads part of the cache back in 16 bits, the draft's
queries attend to it, and the target's verification attends to it and to the
tree's own keys.  The cache holds one signed 8-bit float (4 exponent bits, 3
mantissa bits) per element and one power-of-two exponent for every block of 64
tokens and cached head:

    value[b, h, t, d] = code[b, h, t, d] * 2 ** exp[b, h, t // 64]

Shapes are those of the evaluation workloads and of the bench (Vicuna-7B/13B/33B
and Mistral-7B layers); ``draw`` spreads over the same ranges.  Inputs are random
numbers made on the GPU from the seed; caches, workspaces and output buffers are
kept by the program between calls, as a decoding loop keeps them.
"""
import math
import random

import torch

own = False
_binding = None           # the framework's calls, once `own` has asked for them

BLOCK = 64                # tokens that share an exponent
EXP_MIN, EXP_MAX = -117, 119
TOP = 448.0               # the largest code
CACHE_MOST = 4 * 52 * 16384 * 128 * 2      # codes of the largest cache read
WORKSPACE = 256 << 20     # what a decoding program reserves once for its largest call
ROWS_KEYS_MOST = 4 * 52 * 64 * 16384 * 128
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    attn = dict(D=128, dtype="bf16", len_seed=0)
    return [
        # one draft step of a single user's Vicuna-7B decode: the smallest call, all launch and latency
        dict(attn, name="cross-7b-b1", kind="cross", B=1, H=32, H_kv=32, kv_min=2048, kv_max=2048),
        # the same step with Vicuna-33B heads, four long contexts: the largest of its kind, all HBM
        dict(attn, name="cross-33b-long", kind="cross", B=4, H=52, H_kv=52, kv_min=16384, kv_max=16384),
        # a draft step over a grouped-query target (Mistral-7B: 32 query over 8 cached heads)
        dict(attn, name="cross-mistral-gqa", kind="cross", B=4, H=32, H_kv=8, kv_min=16384, kv_max=16384),
        # verification of a plain gamma = 5 proposal, single user
        dict(attn, name="verify-7b-chain", kind="verify", B=1, H=32, H_kv=32, kv_min=2048, kv_max=2048, n=6,
             depth=5, branch=1),
        # verification in a served batch of ragged contexts, odd lengths
        dict(attn, name="verify-13b-ragged", kind="verify", B=8, H=40, H_kv=40, kv_min=512, kv_max=4096, n=26,
             depth=5, branch=4, len_seed=3),
        # verification of 64-node trees over long contexts
        dict(attn, name="verify-33b-long", kind="verify", B=4, H=52, H_kv=52, kv_min=16384, kv_max=16384, n=64,
             depth=6, branch=6),
        # verification of CaPE-sized trees (32 tokens and the root) on a grouped-query target
        dict(attn, name="verify-mistral-cape", kind="verify", B=4, H=32, H_kv=8, kv_min=16384, kv_max=16384, n=33,
             depth=5, branch=4),
        # the tiny fp32 workload's verification: what small checks and comparisons run in
        dict(name="verify-tiny-f32", kind="verify", B=1, H=4, H_kv=4, D=64, dtype="f32", kv_min=128, kv_max=128,
             len_seed=0, n=5, depth=4, branch=1),
        # the keys and values of four prompts go into a layer's empty cache
        dict(name="append-7b-prompt", kind="append", layers=1, B=4, H_kv=32, D=128, dtype="bf16", kv_min=0, kv_max=0,
             n=2048, rows_min=2048, path=False, len_seed=0),
        # a round's end: the accepted path of a CaPE tree joins the caches of all 32 layers, mid-block
        dict(name="append-7b-accept", kind="append", layers=32, B=1, H_kv=32, D=128, dtype="bf16", kv_min=1996,
             kv_max=1996, n=33, rows_min=5, path=True, len_seed=0),
        # a single user's layer read back for a 16-bit consumer
        dict(name="read-7b-b1", kind="read", layers=1, B=1, H_kv=32, D=128, dtype="bf16", kv_min=2048, kv_max=2048,
             len_seed=0),
        # a grouped-query target's long contexts read back
        dict(name="read-mistral-b4", kind="read", layers=1, B=4, H_kv=8, D=128, dtype="bf16", kv_min=16384,
             kv_max=16384, len_seed=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["cross", "cross", "cross", "verify", "verify", "verify", "verify", "append", "append", "read"])
    H, H_kv = rng.choice([(32, 32), (40, 40), (52, 52), (32, 8), (32, 8), (8, 8), (24, 8)])
    kv = _log_int(rng, 1, 16384) if rng.random() < 0.2 else _log_int(rng, 128, 16384)
    c = dict(kind=kind, B=_log_int(rng, 1, 8), H_kv=H_kv, D=rng.choice([128, 128, 128, 64]), dtype="bf16", kv_max=kv,
             kv_min=rng.choice([kv, max(1, kv // 8)]), len_seed=rng.randrange(1000))
    if kind == "append":
        c["path"] = rng.random() < 0.5
        c["n"] = _log_int(rng, 1, 64) if c["path"] else _log_int(rng, 1, 4096)
        c["rows_min"] = min(c["n"], rng.choice([1, 4, c["n"]]))
        c["layers"] = rng.choice([1, 4, 32]) if c["path"] else 1
        c["kv_max"], c["kv_min"] = min(c["kv_max"], 4096), min(c["kv_min"], rng.choice([0, 4096]))
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c["B"] = min(c["B"], 4)
    elif kind == "read":
        c.update(layers=rng.choice([1, 1, 2]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    else:
        c["H"] = H
        if kind == "verify":
            n = min(_log_int(rng, 1, 64), 256 * H_kv // H)
            c.update(n=n, **(dict(depth=64, branch=1) if n <= 8 else dict(depth=6, branch=6)))
        if rng.random() < 0.1:  # fp32 queries: small checks
            c.update(dtype="f32", H=4, H_kv=rng.choice([4, 2]), B=min(c["B"], 2), kv_max=min(kv, 1024))
            c["kv_min"] = min(c["kv_min"], c["kv_max"])
            c["n"] = min(c.get("n", 1), 16)
            if kind == "cross":
                del c["n"]
    while c["B"] > 1 and c.get("layers", 1) * c["B"] * c["H_kv"] * (c["kv_max"] + c.get("n", 0)) * c["D"] * 2 > CACHE_MOST:
        c["B"] -= 1
    while c.get("layers", 1) * c["B"] * c["H_kv"] * (c["kv_max"] + c.get("n", 0)) * c["D"] * 2 > CACHE_MOST:
        c["kv_max"] = c["kv_max"] * 3 // 4
        c["kv_min"] = min(c["kv_min"], c["kv_max"])
    while c["B"] > 1 and c["B"] * c.get("H", 1) * c.get("n", 1) * c["kv_max"] * c["D"] > ROWS_KEYS_MOST:
        c["B"] -= 1
    while c["B"] > 1 and work(c)["bytes"] > CACHE_MOST:
        c["B"] -= 1
    while work(c)["bytes"] > CACHE_MOST:
        c["kv_max"] = c["kv_max"] * 3 // 4
        c["kv_min"] = min(c["kv_min"], c["kv_max"])
    return c


def _between(c, lo, hi, salt):
    """Lengths of the batch's sequences: part of the case, so that its work is known without the inputs."""
    r = random.Random(c["len_seed"] * 7 + salt)
    return [r.randint(c[lo], c[hi]) for _ in range(c["B"])]


def _lengths(c):
    return _between(c, "kv_min", "kv_max", 0)


def _rows(c):
    """Rows of each sequence that an append adds."""
    return _between(c, "rows_min", "n", 1) if not c["path"] else [min(c["n"], x) for x in _between(
        dict(c, top=max(c["rows_min"], min(c["n"], 6))), "rows_min", "top", 1)]


def _cap(c, extra):
    """Rows of a slab of the cache: room for what comes, and not a multiple of the block."""
    return (c["kv_max"] + extra + 15) // 16 * 16


# ------------------------------------------------------------------ inputs
def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + k)


def _normal(seed, k, shape, dtype):
    return torch.randn(shape, generator=_gen(seed, k), device="cuda", dtype=TYPES[dtype])


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tokens(seed, k, shape, dtype):
    """Keys or values as a model gives them, [..., tokens, D]: channels and tokens of different magnitude."""
    x = torch.randn(shape, generator=_gen(seed, k), device="cuda")
    x *= torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=_gen(seed, k + 50), device="cuda"))
    x *= torch.exp(0.4 * torch.randn(shape[-1], generator=_gen(seed, k + 80), device="cuda"))
    return x.to(TYPES[dtype])


def _exponent(amax):
    """The least e with amax <= 448 * 2**e: 448 = 0.875 * 2**9, amax = m * 2**y with m in [0.5, 1)."""
    m, y = torch.frexp(amax)
    return torch.where(amax > 0, y - 9 + (m > 0.875).int(), torch.full_like(y, EXP_MIN)).clamp(EXP_MIN, EXP_MAX)


def _two_to(e):
    """2 ** e in fp32 for int e, exactly (a power function need not be); what is below the normal range counts as its end."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _codes(x, exp):
    """fp32 x to the nearest codes (ties to even, the largest code at most) for int exponents that broadcast to it."""
    return torch.clamp(x * _two_to(-exp), -TOP, TOP).to(torch.float8_e4m3fn)


def _cache(seed, k, lead, rows, D):
    """Codes [*lead, rows, D] and exponents [*lead, blocks] of a cache filled with tokens, built slab by slab to
    bound what it takes."""
    nb = -(-rows // BLOCK)
    codes = torch.empty(lead + (rows, D), dtype=torch.float8_e4m3fn, device="cuda")
    exps = torch.empty(lead + (nb,), dtype=torch.int8, device="cuda")
    for i in range(lead[0]):
        x = _tokens(seed * 131 + i, k, lead[1:] + (nb * BLOCK, D), "f32").view(lead[1:] + (nb, BLOCK, D))
        e = _exponent(x.abs().amax((-1, -2)))
        codes[i] = _codes(x, e[..., None, None]).view(lead[1:] + (nb * BLOCK, D))[..., :rows, :]
        exps[i] = e.to(torch.int8)
    return codes, exps


def _tree(r, n, depth, branch):
    """Parents of a random tree of n nodes: each node a child of an earlier one with room."""
    parent, level, kids = [-1], [0], [0] * n
    for i in range(1, n):
        p = r.choice([j for j in range(i) if level[j] < depth and kids[j] < branch])
        kids[p] += 1
        parent.append(p)
        level.append(level[p] + 1)
    return parent


def prepare(case, seed):
    c = case
    lens = _lengths(c)
    s = dict(case=c, lens=lens, kv_len=_i32(lens), kv_max=c["kv_max"])
    B, H_kv, D = c["B"], c["H_kv"], c["D"]
    if c["kind"] in ("append", "read"):
        lead = (c["layers"], B, H_kv)
        s["K"], s["K_exp"] = _cache(seed, 1, lead, _cap(c, c.get("n", 0)), D)
        s["V"], s["V_exp"] = _cache(seed, 2, lead, _cap(c, c.get("n", 0)), D)
        if c["kind"] == "read":
            shape = lead + (c["kv_max"], D)
            s["K_out"], s["V_out"] = (torch.empty(shape, dtype=TYPES[c["dtype"]], device="cuda") for _ in range(2))
            return s
        shape = (c["layers"], B, c["n"], H_kv, D)
        s["k"] = _tokens(seed, 3, shape, c["dtype"])
        s["v"] = _tokens(seed, 4, shape, c["dtype"])
        rows = _rows(c)
        s["length"] = _i32([x - 1 for x in rows])
        s["path"] = None
        if c["path"]:  # a root path: increasing nodes from node 0, -1 after its end
            r = random.Random(seed * 41 + 3)
            s["path"] = _i32([[0] + sorted(r.sample(range(1, c["n"]), m - 1)) + [-1] * (c["n"] - m) for m in rows])
        s["new_len"] = torch.empty(B, dtype=torch.int32, device="cuda")
        return s
    rows = _cap(c, BLOCK)
    s["K"], s["K_exp"] = _cache(seed, 1, (B, H_kv), rows, D)
    s["V"], s["V_exp"] = _cache(seed, 2, (B, H_kv), rows, D)
    n = c.get("n", 1)
    s["q"] = _normal(seed, 5, (B, n, c["H"], D), c["dtype"])
    s["out"] = torch.empty((B, n, c["H"], D), dtype=TYPES[c["dtype"]], device="cuda")
    if c["kind"] == "verify":
        s["k"] = _tokens(seed, 3, (B, n, H_kv, D), c["dtype"])
        s["v"] = _tokens(seed, 4, (B, n, H_kv, D), c["dtype"])
        r = random.Random(seed * 31 + 7)
        s["parent"] = _i32([_tree(r, n, c["depth"], c["branch"]) for _ in range(B)])
    s["ws"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the operators, plainly
def _values(codes, exp, rows):
    """fp32 values of the first `rows` rows of a cache."""
    return codes[..., :rows, :].float() * _two_to(exp).repeat_interleave(BLOCK, -1)[..., :rows, None]


def _square(m):
    return (m @ m).clamp(max=1.0)


def _sees(parent):
    """[B, n, n]: whether node j is node i or an ancestor of it (64 levels at most)."""
    B, n = parent.shape
    up = torch.zeros((B, n, n + 1), device=parent.device).scatter_(2, (parent.long() % (n + 1))[..., None], 1.0)[..., :n]
    m = up + torch.eye(n, device=parent.device)
    return _square(_square(_square(_square(_square(_square(m)))))) > 0


def _plain_attention(s):
    c, q = s["case"], s["q"]
    B, n, H, D = q.shape
    H_kv, g = c["H_kv"], H // c["H_kv"]
    S = max(1, s["kv_max"])
    K, V = _values(s["K"], s["K_exp"], S), _values(s["V"], s["V_exp"], S)
    x = q.float().view(B, n, H_kv, g, D).transpose(1, 2).reshape(B, H_kv, n * g, D) / math.sqrt(D)
    ahead = torch.arange(S, device=q.device) >= s["kv_len"][:, None]
    scores = (x @ K.transpose(-1, -2)).masked_fill(ahead[:, None, None, :], -math.inf)
    if c["kind"] == "verify":
        k, v = (s[w].float().transpose(1, 2) for w in ("k", "v"))
        hidden = ~_sees(s["parent"]).repeat_interleave(g, 1)
        scores = torch.cat([scores, (x @ k.transpose(-1, -2)).masked_fill(hidden[:, None], -math.inf)], -1)
        V = torch.cat([V, v], 2)
    top = scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    out = (p @ V) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return out.view(B, H_kv, n, g, D).transpose(1, 2).reshape(B, n, H, D).to(q.dtype)


def _plain_append(s):
    K, V = s["K"], s["V"]
    L, B, H_kv, cap, D = K.shape
    n = s["k"].shape[2]
    nb = s["K_exp"].shape[-1]
    start = s["kv_len"].clamp(0, cap - n)
    rows = s["length"].clamp(-1, n - 1) + 1
    # where each row of the cache comes from: new row (its place from the start), or none
    at = torch.arange(nb * BLOCK, device=K.device) - start[:, None]
    fresh = (at >= 0) & (at < rows[:, None])
    src = at.clamp(0, n - 1)
    if s["path"] is not None:
        src = s["path"].clamp(0, n - 1).gather(1, src).long()
    f = fresh[None, :, None, :, None]
    touched = fresh.view(B, nb, BLOCK).any(-1)
    keeps = touched & (torch.arange(nb, device=K.device) * BLOCK < start[:, None])  # holds rows from before
    kept = ((torch.arange(nb * BLOCK, device=K.device) < start[:, None])
            & keeps.repeat_interleave(BLOCK, 1))[None, :, None, :, None]

    def one(codes, exp, new):
        x = torch.gather(new.float().transpose(2, 3), 3, src[None, :, None, :, None].expand(L, B, H_kv, -1, D))
        size = torch.where(f & x.isfinite(), x.abs(), 0.0).view(L, B, H_kv, nb, BLOCK, D).amax((-1, -2))
        need = _exponent(size)
        old = exp.int()
        e = torch.where(keeps[None, :, None], torch.maximum(need, old), need)
        e = torch.where(touched[None, :, None], e, old)
        per_row = e.repeat_interleave(BLOCK, -1)[..., None]
        was = old.repeat_interleave(BLOCK, -1)[..., None]
        there = torch.nn.functional.pad(codes.view(torch.uint8), (0, 0, 0, nb * BLOCK - cap)).view(torch.float8_e4m3fn)
        again = _codes(there.float(), per_row - was)
        got = torch.where(f, _codes(x, per_row).view(torch.uint8),
                          torch.where(kept, again.view(torch.uint8), there.view(torch.uint8)))
        return got[..., :cap, :].contiguous().view(torch.float8_e4m3fn), e.to(torch.int8)

    (k8, ke), (v8, ve) = one(K, s["K_exp"], s["k"]), one(V, s["V_exp"], s["v"])
    return dict(K=k8, V=v8, K_exp=ke, V_exp=ve, new_len=start + rows)


def _plain_read(s):
    S = s["K_out"].shape[-2]
    past = (torch.arange(S, device=s["K"].device) >= s["kv_len"][:, None])[None, :, None, :, None]
    return tuple(_values(s[w], s[w + "_exp"], S).masked_fill(past, 0.0).to(s[w + "_out"].dtype) for w in ("K", "V"))


def _library():
    global _binding
    if _binding is None:
        from paper_2402_02082_gb300 import binding
        _binding = binding
    return _binding


def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return {"append": _plain_append, "read": _plain_read}.get(kind, _plain_attention)(s)
    lib = _library()
    cache = (s["K"], s["V"], s["K_exp"], s["V_exp"])
    if kind == "append":
        lib.glide_kv8_append(s["k"], s["v"], *cache, s["kv_len"], s["new_len"], s["path"], s["length"])
        return dict(K=s["K"], V=s["V"], K_exp=s["K_exp"], V_exp=s["V_exp"], new_len=s["new_len"])
    if kind == "read":
        return lib.glide_kv8_read(*cache, s["kv_len"], s["K_out"], s["V_out"])
    if kind == "cross":
        return lib.glide_kv8_cross_attn(s["q"], *cache, s["kv_len"], s["kv_max"], s["out"], s["ws"])
    return lib.glide_kv8_verify_attn(s["q"], s["parent"], s["k"], s["v"], *cache, s["kv_len"], s["kv_max"], s["out"],
                                     s["ws"])


# ------------------------------------------------------------------ from the definition, in 64 bits
def _power(e):
    """2 ** e in 64 bits for whole e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_attention(s):
    c = s["case"]
    q = s["q"].double()
    B, n, H, D = q.shape
    g = H // c["H_kv"]
    out = torch.zeros_like(q)
    for b in range(B):
        t = torch.arange(s["lens"][b], device=q.device)
        if c["kind"] == "verify":
            up, mask = s["parent"][b].tolist(), torch.zeros((n, n), dtype=torch.bool)
            for i in range(n):
                j = i
                while j >= 0:
                    mask[i, j] = True
                    j = up[j]
            mask = mask.to(q.device)
        for h in range(H):
            k = h // g
            keys = s["K"][b, k][: len(t)].double() * _power(s["K_exp"][b, k])[t // BLOCK, None]
            vals = s["V"][b, k][: len(t)].double() * _power(s["V_exp"][b, k])[t // BLOCK, None]
            if c["kind"] == "verify":
                keys = torch.cat([keys, s["k"][b, :, k].double()])
                vals = torch.cat([vals, s["v"][b, :, k].double()])
            if len(keys) == 0:
                continue
            sc = q[b, :, h] @ keys.T / D ** 0.5
            if c["kind"] == "verify":
                sc[:, len(t):][~mask] = -math.inf
            out[b, :, h] = torch.softmax(sc, -1) @ vals
    return out


def _nearest(y):
    """The code nearest to y, ties to even: steps of an eighth of y's binade, of 2**-9 below 2**-6."""
    step = _power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return (torch.round(y / step) * step).clamp(-TOP, TOP)


def _exact_append(s):
    n = s["k"].shape[2]
    L, B, H_kv, cap, D = s["K"].shape
    got = dict(new_len=s["kv_len"].clone())
    for w, new in (("K", s["k"]), ("V", s["v"])):
        codes, exp = s[w].double(), s[w + "_exp"].clone()
        for b in range(B):
            start, m = min(max(s["lens"][b], 0), cap - n), int(s["length"][b]) + 1
            nodes = s["path"][b, :m].long() if s["path"] is not None else torch.arange(m, device=codes.device)
            x = new[:, b].double()[:, nodes].transpose(1, 2)                     # [L, H_kv, m, D]
            for blk in range(start // BLOCK, -(-(start + m) // BLOCK)):
                lo, hi = max(start, blk * BLOCK), min(start + m, (blk + 1) * BLOCK)
                part = x[:, :, lo - start: hi - start]
                size = part.abs().amax((-1, -2))
                e = torch.ceil(torch.log2(size.clamp(min=1e-300) / TOP))
                e = e + (size > TOP * _power(e)) - (size <= TOP * _power(e - 1)).double()
                e = e.clamp(EXP_MIN, EXP_MAX)
                if blk * BLOCK < start:
                    was = exp[:, b, :, blk].double()
                    e = torch.maximum(e, was)
                    keep = codes[:, b, :, blk * BLOCK: start]
                    codes[:, b, :, blk * BLOCK: start] = _nearest(keep * _power(was - e)[..., None, None])
                codes[:, b, :, lo:hi] = _nearest(part * _power(-e)[..., None, None])
                exp[:, b, :, blk] = e.to(torch.int8)
            got["new_len"][b] = start + m
        got[w], got[w + "_exp"] = codes, exp
    return got


def _exact_read(s):
    found = []
    for w in ("K", "V"):
        S = s[w + "_out"].shape[-2]
        t = torch.arange(S, device=s[w].device)
        x = s[w][..., :S, :].double() * _power(s[w + "_exp"])[..., t // BLOCK, None]
        for b, m in enumerate(s["lens"]):
            x[:, b, :, m:] = 0.0
        found.append(x)
    return tuple(found)


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "read": _exact_read}.get(case["kind"], _exact_attention)(s)


def work(case):
    c = case
    lens, D, H_kv, size = _lengths(c), c["D"], c["H_kv"], 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "append":  # new rows in, their codes and exponents out
        m, per = sum(_rows(c)), c["layers"] * 2 * H_kv
        return {"bytes": m * per * D * (size + 1) + per * (m // BLOCK + c["B"]) + 8 * c["B"], "flops": m * per * D * 2}
    if c["kind"] == "read":    # codes and exponents in, values (and zeros past a sequence's end) out
        per = c["layers"] * 2 * H_kv
        return {"bytes": sum(lens) * per * (D + 1 / BLOCK) + per * D * size * c["B"] * c["kv_max"] + 4 * c["B"],
                "flops": sum(lens) * per * D}
    n = c.get("n", 1)
    tree = n if c["kind"] == "verify" else 0
    rows = c["B"] * n * c["H"] * D * size
    return {"bytes": sum(lens) * 2 * H_kv * (D + 1 / BLOCK) + 2 * rows
            + tree * c["B"] * (2 * H_kv * D * size + 4) + 4 * c["B"],
            "flops": 4 * D * n * c["H"] * sum(x + tree for x in lens)}
