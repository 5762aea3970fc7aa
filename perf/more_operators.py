"""The cases that the paged cache and the attention of prompts and chunks are measured on.

A serving program that keeps the target's keys and values in pages makes four kinds of call.  A plan gives each
request of a step the pages that its new tokens need and says where every token goes; an append writes the new
keys and values there; chunks of new tokens (one token, a proposal, a part of a prompt) attend to the pages; and
whole prompts, packed one behind the other, attend to themselves.

    pages      K, V [n_pages, H_kv, P, D]; token t of request b is row t % P of page block_table[b, t // P]
    slot       page * P + row, for each new token; -1: the token goes nowhere
    chunk      row i of a request's m new tokens sees its keys t <= kv_len - m + i (kv_len counts the new ones)
    prompt     row i of a sequence sees the sequence's tokens 0 .. i

Shapes are those of the evaluation workloads and of the bench (Vicuna-7B/13B/33B and Mistral-7B layers); ``draw``
spreads over the same ranges.  Inputs are random numbers made on the GPU from the seed; pools, tables, workspaces and
output buffers are kept by the program between calls, as a serving loop keeps them.
"""
import math
import random

import torch

own = False
_binding = None           # the framework's calls, once `own` has asked for them

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
WORKSPACE = 512 << 20     # what a serving program reserves once for its largest call
SCORES = 1 << 28          # scores that the plain form of a prompt holds at a time
PAIRS_MOST = 32 * 16384 * 8192 * 128       # heads x visible (query, key) pairs x D of the largest prompt
BYTES_MOST = 2 * 2 * 16384 * 32 * 128 * 2  # of the largest append
CACHE_MOST = 2 * 4 * 52 * 16384 * 128 * 2  # keys and values of the largest cache that is read
SCORES_MOST = 8 * 40 * 512 * 4096          # padded scores of the largest chunk


def listed():
    return [
        # a decoding step of a small served batch: one token each, now and then a new page; all launch and latency
        dict(name="plan-decode-b32", kind="plan", B=32, P=16, q_max=1, kv_max=4096, finished=0.05, spare=1.0, len_seed=1),
        # a step that mixes chunks of prompts with decoding requests, in a pool that runs short
        dict(name="plan-mixed-b1024", kind="plan", B=1024, P=16, q_max=512, kv_max=4096, finished=0.1, spare=0.9,
             len_seed=2),
        # the keys and values of a decoding step of 64 requests join a grouped-query target's layer
        dict(name="append-mistral-b64", kind="append", T=64, H=32, H_kv=8, D=128, P=16, dtype="bf16", skipped=0.0,
             fused=True, len_seed=3),
        # those of eight prompts of 2048 tokens, straight from a fused projection's output
        dict(name="append-7b-prompts", kind="append", T=16384, H=32, H_kv=32, D=128, P=16, dtype="bf16", skipped=0.0,
             fused=True, len_seed=4),
        # one token of a single user's Vicuna-7B decode: the smallest attention call
        dict(name="token-7b-b1", kind="paged", B=1, H=32, H_kv=32, D=128, P=16, dtype="bf16", q_max=1, q_min=1,
             kv_min=2048, kv_max=2048, len_seed=5),
        # one token each of a served batch of ragged contexts on a grouped-query target: all HBM
        dict(name="token-mistral-b32", kind="paged", B=32, H=32, H_kv=8, D=128, P=16, dtype="bf16", q_max=1, q_min=1,
             kv_min=1024, kv_max=16384, len_seed=6),
        # a chain proposal of five tokens and the last one verified over four long contexts, Vicuna-33B heads
        dict(name="chain-33b-long", kind="paged", B=4, H=52, H_kv=52, D=128, P=64, dtype="bf16", q_max=6, q_min=6,
             kv_min=16384, kv_max=16384, len_seed=7),
        # chunks of prompts of odd lengths beside decoding requests, Vicuna-13B heads
        dict(name="chunk-13b-ragged", kind="paged", B=8, H=40, H_kv=40, D=128, P=32, dtype="bf16", q_max=512, q_min=1,
             kv_min=512, kv_max=4096, len_seed=8),
        # two small prompts in fp32: what small checks and comparisons run in
        dict(name="prompt-tiny-f32", kind="prompt", B=2, H=4, H_kv=4, D=64, dtype="f32", len_min=60, len_max=128,
             pad=3, fused=False, len_seed=9),
        # many short prompts of odd lengths in one pack, Vicuna-33B heads, a padded pack
        dict(name="prompt-33b-short", kind="prompt", B=24, H=52, H_kv=52, D=128, dtype="bf16", len_min=1, len_max=333,
             pad=100, fused=True, len_seed=10),
        # four Vicuna-7B prompts that fill the context
        dict(name="prompt-7b-full", kind="prompt", B=4, H=32, H_kv=32, D=128, dtype="bf16", len_min=2048, len_max=2048,
             pad=0, fused=True, len_seed=11),
        # a long prompt on a grouped-query target
        dict(name="prompt-mistral-long", kind="prompt", B=1, H=32, H_kv=8, D=128, dtype="bf16", len_min=16384,
             len_max=16384, pad=0, fused=True, len_seed=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "paged", "paged", "paged", "paged", "prompt", "prompt", "prompt", "prompt"])
    H, H_kv = rng.choice([(32, 32), (40, 40), (52, 52), (32, 8), (32, 8), (8, 8), (24, 8), (8, 1)])
    c = dict(kind=kind, P=rng.choice([16, 16, 32, 64, 128]), len_seed=rng.randrange(1000))
    if kind == "plan":
        c.update(B=_log_int(rng, 1, 1024), q_max=_log_int(rng, 1, 512), kv_max=_log_int(rng, 16, 4096),
                 finished=rng.choice([0.0, 0.1, 0.3]), spare=rng.choice([0.5, 0.9, 1.0, 1.0]))
        return c
    c.update(H=H, H_kv=H_kv, D=rng.choice([128, 128, 128, 64]), dtype="bf16")
    if kind == "append":
        c.update(T=_log_int(rng, 1, 16384), dtype=rng.choice(["bf16", "bf16", "f32"]),
                 skipped=rng.choice([0.0, 0.0, 0.2]), fused=rng.random() < 0.5)
        while work(c)["bytes"] > BYTES_MOST:
            c["T"] = c["T"] * 3 // 4
        return c
    small = rng.random() < 0.15
    if small:  # fp32: small checks
        c.update(dtype="f32", H=4, H_kv=rng.choice([4, 2, 1]))
    if kind == "prompt":
        del c["P"]
        c.update(B=_log_int(rng, 1, 2 if small else 32), len_max=_log_int(rng, 1, 256 if small else 8192),
                 pad=rng.choice([0, 0, 5, 77]), fused=rng.random() < 0.7)
        c["len_min"] = max(1, c["len_max"] // rng.choice([1, 4, 100]))
        while c["B"] > 1 and (work(c)["flops"] > 4 * PAIRS_MOST or sum(_lengths(c)) > 32768):
            c["B"] -= 1
        while work(c)["flops"] > 4 * PAIRS_MOST:
            c["len_max"] = c["len_max"] * 3 // 4
            c["len_min"] = min(c["len_min"], c["len_max"])
        return c
    kv = _log_int(rng, 1, 1024 if small else 16384)
    c.update(B=_log_int(rng, 1, 2 if small else 64), q_max=_log_int(rng, 1, min(kv, 16 if small else 512)), kv_max=kv)
    c["q_min"] = rng.choice([1, c["q_max"]])
    c["kv_min"] = max(c["q_max"], rng.choice([kv, kv // 8]))
    while c["B"] > 1 and (c["B"] * c["H"] * c["q_max"] * kv > SCORES_MOST or work(c)["bytes"] > CACHE_MOST):
        c["B"] -= 1
    while c["B"] * c["H"] * c["q_max"] * kv > SCORES_MOST:
        c["q_max"] = c["q_max"] * 3 // 4
        c["q_min"] = min(c["q_min"], c["q_max"])
    return c


def _between(c, lo, hi, salt):
    """Lengths of the batch's sequences: part of the case, so that its work is known without the inputs."""
    r = random.Random(c["len_seed"] * 7 + salt)
    return [r.randint(lo, hi) for _ in range(c["B"])]


def _lengths(c):
    return _between(c, c["len_min"], c["len_max"], 0)


def _chunks(c):
    """New tokens of each request (short ones more often, as decoding requests are) and tokens with them."""
    r = random.Random(c["len_seed"] * 7 + 1)
    m = [r.choice([c["q_min"], c["q_max"], r.randint(c["q_min"], c["q_max"])]) for _ in range(c["B"])]
    return m, _between(c, c["kv_min"], c["kv_max"], 2)


def _requests(c):
    """New tokens (-1: the request has finished), tokens in the cache and pages held of each request of a step."""
    r = random.Random(c["len_seed"] * 7 + 3)
    q, kv, held = [], [], []
    for _ in range(c["B"]):
        q.append(-1 if r.random() < c["finished"] else r.choice([1, 1, r.randint(1, c["q_max"])]))
        kv.append(r.randint(0, c["kv_max"]))
        held.append(-(-kv[-1] // c["P"]) + r.choice([0, 0, 0, 1]))
    return q, kv, held


def _table_width(c):
    return -(-(c["kv_max"] + c["q_max"]) // c["P"]) + 1


def _pages_needed(c):
    q, kv, held = _requests(c)
    return sum(max(0, -(-(k + m) // c["P"]) - h) for m, k, h in zip(q, kv, held) if m > 0)


# ------------------------------------------------------------------ inputs
def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed(seed * 1009 + k)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tokens(seed, k, shape, dtype):
    """Keys or values as a model gives them, [tokens, ..., D]: channels of different magnitude."""
    x = torch.randn(shape, generator=_gen(seed, k), device="cuda")
    x *= torch.exp(0.4 * torch.randn(shape[-1], generator=_gen(seed, k + 80), device="cuda"))
    return x.to(TYPES[dtype])


def _projected(seed, c, T):
    """q [T, H, D] and k, v [T, H_kv, D] of T tokens: parts of one projection's rows, or tensors of their own."""
    H, H_kv, D = c["H"], c["H_kv"], c["D"]
    x = _tokens(seed, 1, (T, H + 2 * H_kv, D), c["dtype"])
    parts = x[:, :H], x[:, H: H + H_kv], x[:, H + H_kv:]
    return parts if c["fused"] else tuple(p.contiguous() for p in parts)


def _pool(seed, c, pages):
    return tuple(_tokens(seed, k, (pages, c["H_kv"], c["P"], c["D"]), c["dtype"]) for k in (2, 3))


def _offsets(lens):
    return _i32([0] + list(torch.tensor(lens).cumsum(0)))


def prepare(case, seed):
    c = case
    s = dict(case=c)
    if c["kind"] == "plan":
        q, kv, held = _requests(c)
        B, width = c["B"], _table_width(c)
        n_pages = sum(held) + int(_pages_needed(c) * c["spare"])
        ids = torch.randperm(max(1, n_pages), generator=_gen(seed, 1), device="cuda").int()
        table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        s["held"] = _i32(held)
        there = torch.arange(width, device="cuda") < s["held"][:, None]
        table[there] = ids[: sum(held)]
        free = torch.full((len(ids),), -1, dtype=torch.int32, device="cuda")
        free[: n_pages - sum(held)] = ids[sum(held): n_pages]
        T = sum(max(0, m) for m in q) + 7      # a padded step: rows behind the last token
        s.update(q_len=_i32(q), kv_len=_i32(kv), table=table, free=free, n_free=_i32([n_pages - sum(held)]), T=T,
                 cu_q=_i32([0] * (B + 1)), slots=_i32([0] * T), positions=_i32([0] * T), new_kv=_i32([0] * B),
                 new_held=_i32([0] * B), new_free=_i32([0]))
        return s
    if c["kind"] == "append":
        T, P = c["T"], c["P"]
        pages = -(-T // P) + 3
        _, s["k"], s["v"] = _projected(seed, c, T)
        s["K"], s["V"] = _pool(seed, c, pages)
        slots = torch.randperm(pages, generator=_gen(seed, 4), device="cuda")[:, None] * P
        slots = (slots + torch.arange(P, device="cuda")).reshape(-1)[:T]
        off = torch.rand(T, generator=_gen(seed, 5), device="cuda") < c["skipped"]
        s["slots"] = torch.where(off, -1, slots).int()
        return s
    if c["kind"] == "paged":
        m, kv = _chunks(c)
        B, T, P = c["B"], sum(m), c["P"]
        width = -(-c["kv_max"] // P)
        held = [-(-x // P) for x in kv]
        ids = torch.randperm(sum(held) + 1, generator=_gen(seed, 4), device="cuda").int()
        s["table"] = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        s["table"][torch.arange(width, device="cuda") < _i32(held)[:, None]] = ids[: sum(held)]
        s["K"], s["V"] = _pool(seed, c, len(ids))
        s["q"] = _tokens(seed, 1, (T, c["H"], c["D"]), c["dtype"])
        s.update(m=m, kv=kv, cu_q=_offsets(m), kv_len=_i32(kv))
    else:
        s["lens"] = _lengths(c)
        T = sum(s["lens"]) + c["pad"]
        s["q"], s["k"], s["v"] = _projected(seed, c, T)
        s["cu"] = _offsets(s["lens"])
    s["out"] = torch.zeros((T, c["H"], c["D"]), dtype=TYPES[c["dtype"]], device="cuda")
    s["ws"] = torch.zeros(WORKSPACE, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the operators, plainly
def _plain_plan(s):
    P, T, table, free = s["case"]["P"], s["T"], s["table"], s["free"]
    B, width = table.shape
    cols = torch.arange(width, device=table.device)
    ends = s["q_len"].clamp(min=0).cumsum(0).clamp(max=T)
    cu = torch.cat([ends.new_zeros(1), ends])
    m = cu[1:] - cu[:-1]
    done = s["q_len"] < 0
    held = s["held"].long()
    back = torch.where(done, held, 0)
    # pages of finished requests go on top of the stack, in their order
    given = done[:, None] & (cols < held[:, None])
    at = s["n_free"] + (back.cumsum(0) - back)[:, None] + cols
    spill = torch.cat([free, free.new_zeros(1)])
    spill = spill.scatter(0, torch.where(given, at, len(free)).reshape(-1), table.reshape(-1))
    free.copy_(spill[:-1])
    avail = s["n_free"].long() + back.sum()
    want = -(-(s["kv_len"] + m) // P)
    fits = (want <= width) & ~done
    need = torch.where(fits & (m > 0), (want - held).clamp(min=0), 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= avail))
    got = torch.where(ok, need, 0)
    first = held[:, None]
    fresh = (cols >= first) & (cols < first + got[:, None])
    from_top = avail - 1 - ((upto - need)[:, None] + cols - first)
    table.copy_(torch.where(fresh, free[from_top.clamp(0, len(free) - 1)], table))
    row = torch.arange(T, device=table.device)
    b = torch.searchsorted(cu[1:].contiguous(), row, right=True).clamp(max=B - 1)
    real = row < cu[-1]
    pos = s["kv_len"].long()[b] + row - cu[b]
    page = table[b, (pos // P).clamp(0, width - 1)]
    slots = torch.where(real & ok[b], page * P + pos % P, -1)
    return dict(table=table, free=free, cu_q=cu.int(), slots=slots.int(), positions=torch.where(real, pos, 0).int(),
                new_kv=torch.where(done, 0, s["kv_len"] + torch.where(ok, m, 0)).int(),
                new_held=torch.where(done, 0, held + got).int(), new_free=(avail - got.sum()).int().view(1))


def _plain_append(s):
    P = s["K"].shape[2]
    there = s["slots"] >= 0
    slot = s["slots"][there].long()
    s["K"][slot // P, :, slot % P] = s["k"][there]
    s["V"][slot // P, :, slot % P] = s["v"][there]
    return dict(K=s["K"], V=s["V"])


def _weighted(scores, V):
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - top.clamp(min=-1e30))
    return (p @ V) / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_paged(s):
    c, q = s["case"], s["q"]
    T, H, D = q.shape
    B, width = s["table"].shape
    n, H_kv, P, dev = c["q_max"], c["H_kv"], c["P"], q.device
    g, S = H // H_kv, width * P
    m = (s["cu_q"][1:] - s["cu_q"][:-1])[:, None]
    i = torch.arange(n, device=dev)
    rows = torch.where(i < m, s["cu_q"][:-1, None] + i, T)          # where each row of the padded batch lies
    x = torch.cat([q, q.new_zeros(1, H, D)])[rows].float() / math.sqrt(D)
    x = x.view(B, n, H_kv, g, D).transpose(1, 2).reshape(B, H_kv, n * g, D)
    K, V = (s[w][s["table"].clamp(min=0)].transpose(1, 2).reshape(B, H_kv, S, D).float() for w in ("K", "V"))
    sees = s["kv_len"][:, None] - m + 1 + i                         # keys that a row sees
    hidden = torch.arange(S, device=dev) >= sees.repeat_interleave(g, 1)[..., None]
    scores = (x @ K.transpose(-1, -2)).masked_fill(hidden[:, None], -math.inf)
    y = _weighted(scores, V).view(B, H_kv, n, g, D).transpose(1, 2).reshape(B * n, H, D)
    out = s["out"]
    out[rows.reshape(-1)[(i < m).reshape(-1)]] = y[(i < m).reshape(-1)].to(out.dtype)
    return out


def _plain_prompt(s):
    q, k, v, out = s["q"], s["k"], s["v"], s["out"]
    H, H_kv, D = q.shape[1], k.shape[1], q.shape[2]
    g, at = H // H_kv, 0
    for n in s["lens"]:
        K, V = (x[at: at + n].float().transpose(0, 1) for x in (k, v))
        step = max(1, SCORES // (H * n))
        for i in range(0, n, step):  # as many rows at a time as there is room for their scores
            e = min(n, i + step)
            x = q[at + i: at + e].float().view(e - i, H_kv, g, D).transpose(0, 1).reshape(H_kv, -1, D) / math.sqrt(D)
            sees = torch.arange(i, e, device=q.device).repeat_interleave(g)[:, None]
            hidden = torch.arange(e, device=q.device) > sees
            y = _weighted((x @ K[:, :e].transpose(-1, -2)).masked_fill(hidden, -math.inf), V[:, :e])
            out[at + i: at + e] = y.view(H_kv, e - i, g, D).transpose(0, 1).reshape(e - i, H, D).to(out.dtype)
        at += n
    return out


def _library():
    global _binding
    if _binding is None:
        from paper_2402_02082_gb300 import binding
        _binding = binding
    return _binding


def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"plan": _plain_plan, "append": _plain_append, "paged": _plain_paged, "prompt": _plain_prompt}[c["kind"]](s)
    lib = _library()
    if c["kind"] == "plan":
        lib.glide_page_plan(s["q_len"], s["kv_len"], s["held"], s["table"], s["free"], s["n_free"], c["P"], s["cu_q"],
                            s["slots"], s["new_kv"], s["new_held"], s["new_free"], s["positions"])
        return {w: s[w] for w in ("table", "free", "cu_q", "slots", "positions", "new_kv", "new_held", "new_free")}
    if c["kind"] == "append":
        lib.glide_paged_append(s["k"], s["v"], s["K"], s["V"], s["slots"])
        return dict(K=s["K"], V=s["V"])
    if c["kind"] == "paged":
        return lib.glide_paged_attn(s["q"], s["K"], s["V"], s["table"], s["cu_q"], c["q_max"], s["kv_len"], c["kv_max"],
                                    s["out"], s["ws"])
    return lib.glide_prompt_attn(s["q"], s["k"], s["v"], s["cu"], c["len_max"], s["out"], s["ws"])


# ------------------------------------------------------------------ from the definition, in 64 bits
def _exact_plan(s):
    c = s["case"]
    P, T = c["P"], s["T"]
    q, kv, held = _requests(c)
    table, stack = s["table"].tolist(), s["free"].tolist()
    n = int(s["n_free"][0])
    cu, slots, positions, new_kv, new_held = [0], [-1] * T, [0] * T, [], []
    for b, m in enumerate(q):
        if m < 0:
            for page in table[b][: held[b]]:
                stack[n] = page
                n += 1
    asked, top = 0, n
    for b, m in enumerate(q):
        m = max(0, m)
        cu.append(cu[-1] + m)
        if q[b] < 0:
            new_kv.append(0)
            new_held.append(0)
            continue
        need = max(0, -(-(kv[b] + m) // P) - held[b]) if m else 0
        asked += need
        admitted = need == 0 or asked <= top
        if admitted:
            for j in range(need):
                n -= 1
                table[b][held[b] + j] = stack[n]
        for i in range(m):
            t = kv[b] + i
            positions[cu[b] + i] = t
            if admitted:
                slots[cu[b] + i] = table[b][t // P] * P + t % P
        new_kv.append(kv[b] + m * admitted)
        new_held.append(held[b] + need * admitted)
    return dict(table=_i32(table), free=_i32(stack), cu_q=_i32(cu), slots=_i32(slots), positions=_i32(positions),
                new_kv=_i32(new_kv), new_held=_i32(new_held), new_free=_i32([n]))


def _exact_append(s):
    slots = s["slots"].tolist()
    last = {x: i for i, x in enumerate(slots) if x >= 0}
    n_pages, _, P, _ = s["K"].shape
    source = torch.tensor([last.get(x, -1) for x in range(n_pages * P)], device=s["K"].device).view(n_pages, 1, P, 1)
    found = {}
    for w in ("K", "V"):
        new = s[w.lower()].double()[source.clamp(min=0).view(n_pages, P)].transpose(1, 2)
        found[w] = torch.where(source >= 0, new, s[w].double())
    return found


def _exact_paged(s):
    c = s["case"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["q"].device)
    g, at = c["H"] // c["H_kv"], 0
    for b, (m, kv) in enumerate(zip(s["m"], s["kv"])):
        t = torch.arange(kv, device=out.device)
        page, row = s["table"][b].long()[t // c["P"]], t % c["P"]
        last = kv - m + torch.arange(m, device=out.device)
        for h in range(c["H"]):
            keys, vals = (s[w][page, h // g, row].double() for w in ("K", "V"))
            sc = s["q"][at: at + m, h].double() @ keys.T / c["D"] ** 0.5
            out[at: at + m, h] = torch.softmax(torch.where(t > last[:, None], -math.inf, sc), -1) @ vals
        at += m
    return out


def _exact_prompt(s):
    c = s["case"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["q"].device)
    g, at = c["H"] // c["H_kv"], 0
    for n in s["lens"]:
        for h in range(c["H"]):
            q, k, v = (s[w][at: at + n, j].double() for w, j in (("q", h), ("k", h // g), ("v", h // g)))
            for i in range(0, n, 4096):
                sc = q[i: i + 4096] @ k[: i + 4096].T / c["D"] ** 0.5
                after = torch.ones_like(sc, dtype=torch.bool).triu(i + 1)
                out[at + i: min(at + n, at + i + 4096), h] = torch.softmax(sc.masked_fill_(after, -math.inf), -1) @ v[: i + 4096]
        at += n
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "paged": _exact_paged, "prompt": _exact_prompt}[case["kind"]](s)


def work(case):
    c = case
    if c["kind"] == "plan":
        q, kv, held = _requests(c)
        T = sum(max(0, m) for m in q) + 7
        moved = _pages_needed(c) * c["spare"] + sum(h for m, h in zip(q, held) if m < 0)
        used = sum(-(-(k + m) // c["P"]) - k // c["P"] for m, k in zip(q, kv) if m > 0)   # pages that slots lie in
        return {"bytes": 4 * (c["B"] * 6 + 1 + 2 * T + 2 * moved + used), "flops": 0}
    size = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "append":  # each row in and out, and its slot
        return {"bytes": c["T"] * (4 + (1 - c["skipped"]) * 2 * 2 * c["H_kv"] * c["D"] * size), "flops": 0}
    if c["kind"] == "prompt":
        lens = _lengths(c)
        T, pairs, tables = sum(lens), sum(n * (n + 1) // 2 for n in lens), 4 * (c["B"] + 1)
        kept = T
    else:
        m, kv = _chunks(c)
        T, kept = sum(m), sum(kv)
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(m, kv))
        tables = 4 * (2 * c["B"] + 1 + sum(-(-k // c["P"]) for k in kv))
    return {"bytes": 2 * kept * c["H_kv"] * c["D"] * size + 2 * T * c["H"] * c["D"] * size + tables,
            "flops": 4 * c["D"] * c["H"] * pairs}
