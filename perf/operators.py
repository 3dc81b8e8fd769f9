"""Cases, plain forms and 64-bit definitions of the rollout and policy operators.

Four operators that stand around the credit-assignment scans when the policy is a token model:

  sample   actions drawn from logits with temperature, top-k, min-p and top-p, one given uniform a row
  policy   log-probability, entropy and policy loss of given actions, and the loss's gradient
  attend   attention of one query a trajectory over the paged cache of its group's prompt and its own
  tables   page tables, slot maps and positions of a step, built from the trajectories' lengths

``run`` computes the plain form with elementary torch operations where ``own`` is false, and calls
the package's operators where it is true.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WEIGHT_ONE = 2.0 ** 31          # weight of the most likely action: exp(0) in units of 2^-31


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one trajectory waits for its next token: latency
        {"name": "sample one row", "op": "sample", "rows": 1, "actions": 131072, "dtype": "bf16", "pad": 0, "filters": "both", "masked": False},
        # a rollout batch whose trajectories ask for different settings
        {"name": "sample a batch", "op": "sample", "rows": 256, "actions": 131072, "dtype": "bf16", "pad": 0, "filters": "mixed", "masked": False},
        # odd width, padded rows, float32, disallowed actions; some rows allow nothing at all
        {"name": "sample masked odd rows", "op": "sample", "rows": 67, "actions": 50021, "dtype": "f32", "pad": 11, "filters": "mixed", "masked": True},
        # a vector of simulators with a small discrete action set
        {"name": "sample small sets", "op": "sample", "rows": 262144, "actions": 18, "dtype": "f32", "pad": 0, "filters": "none", "masked": False},
        # the learner's batch of such simulators, V-trace advantages and an entropy bonus
        {"name": "policy small sets", "op": "policy", "rows": 1048576, "actions": 18, "dtype": "f32", "pad": 0, "clipped": False, "padding": False},
        # a token policy's minibatch
        {"name": "policy large set", "op": "policy", "rows": 4096, "actions": 131072, "dtype": "bf16", "pad": 0, "clipped": False, "padding": False},
        # clipped loss, odd width, padding tokens between the trajectories
        {"name": "policy padded odd rows", "op": "policy", "rows": 1021, "actions": 50021, "dtype": "bf16", "pad": 0, "clipped": True, "padding": True},
        # one trajectory right after its prompt: latency
        {"name": "attend one row", "op": "attend", "groups": 1, "rows": 1, "heads": 8, "kv_heads": 8, "dim": 64, "page": 16, "prefix": 100, "own": 1},
        # sixteen prompts with eight rollouts each, at all stages
        {"name": "attend sixteen groups", "op": "attend", "groups": 16, "rows": 128, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "prefix": 2048, "own": 2048},
        # one long prompt with many rollouts, early on
        {"name": "attend one long prompt", "op": "attend", "groups": 1, "rows": 256, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "prefix": 32768, "own": 512},
        # every step of generation: one token a trajectory
        {"name": "tables one token", "op": "tables", "rows": 128, "page": 64, "cached": 4096, "added": 1},
        # a new batch of prompts, nothing cached
        {"name": "tables prompts", "op": "tables", "rows": 2048, "page": 16, "cached": 0, "added": 2048},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "policy", "attend", "tables"])
    if op == "sample":
        actions = _log_int(rng, 2, 262144)
        return {"op": op, "rows": _log_int(rng, 1, min(262144, (1 << 25) // actions)), "actions": actions,
                "dtype": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 1, 8, 13]),
                "filters": rng.choice(["none", "both", "mixed"]), "masked": rng.random() < 0.3}
    if op == "policy":
        actions = _log_int(rng, 2, 262144)
        return {"op": op, "rows": _log_int(rng, 1, min(1048576, (1 << 27) // actions)), "actions": actions,
                "dtype": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 1, 8, 13]),
                "clipped": rng.random() < 0.5, "padding": rng.random() < 0.5}
    if op == "attend":
        heads, kv_heads = rng.choice([(8, 8), (16, 2), (32, 8), (28, 4), (20, 1), (32, 32)])
        rows = _log_int(rng, 1, 256)
        most = (1 << 24) // (rows * kv_heads)              # of one trajectory's own tokens
        return {"op": op, "groups": _log_int(rng, 1, min(rows, 32)), "rows": rows, "heads": heads, "kv_heads": kv_heads,
                "dim": rng.choice([64, 128]), "page": rng.choice([16, 32, 64, 128]),
                "prefix": _log_int(rng, 1, (1 << 18) // kv_heads // 8), "own": _log_int(rng, 1, max(1, min(4096, most // 16)))}
    rows = _log_int(rng, 1, 16384)
    return {"op": op, "rows": rows, "page": rng.choice([1, 16, 32, 64, 100]), "cached": rng.choice([0, _log_int(rng, 1, 8192)]),
            "added": rng.choice([1, _log_int(rng, 1, max(1, min(8192, (1 << 22) // rows)))])}


# ------------------------------------------------------------------------------------------ inputs
def _logits(case, g):
    """Rows as a trained policy gives them: a broad bulk and a few strong candidates; `pad` more columns in memory."""
    R, A, dt = case["rows"], case["actions"], DTYPES[case["dtype"]]
    x = torch.empty(R, A + case["pad"], dtype=dt, device=DEV).normal_(0.0, 2.0, generator=g)
    strong = torch.randint(0, A, (R, min(A, 24)), generator=g, device=DEV)
    x.scatter_reduce_(1, strong, (torch.rand(strong.shape, generator=g, device=DEV) * 8 + 6).to(dt), "amax")
    return x[:, :A]


def _log_softmax_at(x, actions, temperature):
    """log-probability of the given actions, a block of rows at a time."""
    got = []
    for k in range(0, x.shape[0], 65536 if x.shape[1] < 1024 else 256):
        f = x[k:k + (65536 if x.shape[1] < 1024 else 256)].float() / temperature
        got.append(f.gather(1, actions[k:k + f.shape[0], None].long())[:, 0] - torch.logsumexp(f, 1))
    return torch.cat(got)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op = case["op"]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    def ints(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.int32)

    if op == "sample":
        R, A = case["rows"], case["actions"]
        x = _logits(case, g)
        if case["masked"]:
            off = rand(R, A) < 0.4
            x[off] = -math.inf
            x[off & (rand(R, A) < 0.5)] = torch.finfo(x.dtype).min
            x[::16] = -math.inf
        s = {"op": op, "logits": x, "uniforms": rand(R), "temperature": None, "top_k": None, "top_p": None, "min_p": None}
        if case["filters"] == "both":
            s |= {"temperature": torch.full((R,), 0.8, device=DEV), "top_k": torch.full((R,), 50, dtype=torch.int32, device=DEV),
                  "top_p": torch.full((R,), 0.9, device=DEV)}
        elif case["filters"] == "mixed":       # a fifth of the rows greedy, every filter on about half of them
            t, k = rand(R) * 1.2 + 0.3, ints(1, 200, (R,))
            s |= {"temperature": torch.where(rand(R) < 0.2, torch.zeros_like(t), t), "top_k": torch.where(rand(R) < 0.5, torch.zeros_like(k), k),
                  "top_p": torch.where(rand(R) < 0.5, torch.ones_like(t), rand(R) * 0.5 + 0.5),
                  "min_p": torch.where(rand(R) < 0.5, torch.zeros_like(t), rand(R) * 0.1)}
        return s
    if op == "policy":
        R, A = case["rows"], case["actions"]
        x = _logits(case, g)
        s = {"op": op, "logits": x, "actions": ints(0, A, (R,)), "advantages": torch.randn(R, generator=g, device=DEV),
             "old_log_probs": None, "mask": None, "temperature": 0.9, "clip": 0.2, "entropy_coef": 0.01, "scale": 1.0 / R}
        if case["clipped"]:                    # most tokens close to the acting policy, a few stale ones far off
            near, far = rand(R) * 0.3 - 0.15, (rand(R) * 0.3 + 0.3) * torch.where(rand(R) < 0.5, -1.0, 1.0)
            s["old_log_probs"] = _log_softmax_at(x, s["actions"], 0.9) + torch.where(rand(R) < 0.1, far, near)
        if case["padding"]:
            s["mask"] = rand(R) < 0.85
        return s
    if op == "attend":
        Gn, B, H, Hk, D, page = (case[k] for k in ("groups", "rows", "heads", "kv_heads", "dim", "page"))
        # ragged prompts and trajectories, the longest as long as the case says
        pre, mine = ints(case["prefix"] // 2, case["prefix"] + 1, (Gn,)), ints(0, case["own"] + 1, (B,))
        pre[0], mine[-1] = case["prefix"], case["own"]
        cut = torch.sort(torch.randperm(B - 1, generator=g, device=DEV)[:Gn - 1] + 1).values if Gn > 1 else torch.zeros(0, device=DEV)
        offsets = torch.cat([torch.zeros(1, device=DEV), cut, torch.full((1,), B, device=DEV)]).to(torch.int32)
        wp, wb = -(-case["prefix"] // page), -(-case["own"] // page)
        pages = Gn * wp + B * wb + 3
        ids = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        kv = torch.empty(2, pages, page, Hk, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        q = torch.empty(B, H, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        return {"op": op, "q": q, "k": kv[0], "v": kv[1], "prefix_table": ids[:Gn * wp].view(Gn, wp), "prefix_lens": pre,
                "group_offsets": offsets, "block_table": ids[Gn * wp:Gn * wp + B * wb].view(B, wb), "lens": mine,
                "scale": 1.0 / math.sqrt(D), "max_prefix": case["prefix"], "max_len": case["own"],
                "most": int((offsets[1:] - offsets[:-1]).max())}
    B, page = case["rows"], case["page"]
    cached = ints(0, case["cached"] + 1, (B,))
    # lengths of every size whose sum is the same for every seed: pairs that add up to the longest
    added = torch.ones_like(cached)
    if case["added"] > 1:
        half = ints(0, case["added"] + 1, (B // 2,))
        added = torch.cat([half, case["added"] - half, torch.full((B % 2,), case["added"] // 2, dtype=torch.int32, device=DEV)])
        added = added[torch.randperm(B, generator=g, device=DEV)]
    width = -(-(case["cached"] + case["added"]) // page)
    have = (cached + page - 1) // page
    need = int(((cached + added + page - 1) // page).sum())
    ids = torch.randperm(need + 7, generator=g, device=DEV).to(torch.int32)
    held = int(have.sum())
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV)[None, :] < have[:, None]] = ids[:held]
    return {"op": op, "cached": cached, "added": added, "free": ids[held:], "table": table, "page": page, "slots": int(added.sum())}


# ------------------------------------------------------------------------------------------ plain forms
def _plain_sample(s):
    x = s["logits"].float()
    R, A = x.shape
    dev = x.device
    one = torch.ones(R, device=dev)
    t = one if s["temperature"] is None else s["temperature"]
    k = torch.full((R,), A, device=dev) if s["top_k"] is None else s["top_k"].long()
    p = one if s["top_p"] is None else s["top_p"]
    low = one * 0 if s["min_p"] is None else s["min_p"]
    greedy = ~(t > 0)
    inv = 1.0 / torch.where(greedy, one, t)
    top = x.amax(1, keepdim=True)
    e = torch.exp(torch.where(x == top, 0.0, (x - top) * inv[:, None]))
    e = torch.where(top == -math.inf, 0.0, e)
    w = torch.floor(e.double() * WEIGHT_ONE + 0.5).long()                     # whole weights: sums are exact in any order
    order = torch.sort(x, dim=1, descending=True, stable=True).indices        # equal values: the lowest index first
    ws, es = w.gather(1, order), e.gather(1, order)
    rank = torch.arange(A, device=dev)[None, :]
    limit = torch.where(greedy, 1, torch.where(k > 0, k, A))
    keep = (rank < limit[:, None]) & ((rank == 0) | ~(low > 0)[:, None] | (es >= low[:, None]))
    ws = torch.where(keep, ws, 0)
    before = torch.cumsum(ws, 1) - ws
    keep &= (rank == 0) | ~(p < 1)[:, None] | (before.double() < p.double()[:, None] * ws.sum(1, keepdim=True).double())
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0))
    total = kept.sum(1)
    target = torch.minimum(torch.floor(s["uniforms"].double() * total.double()).long(), total - 1)
    actions = (torch.cumsum(kept, 1) <= target[:, None]).sum(1).clamp(max=A - 1)
    none = top[:, 0] == -math.inf
    d = torch.where(x == top, 0.0, (x - top) * inv[:, None]).gather(1, actions[:, None])[:, 0].double()
    full = d - torch.log(w.sum(1).double() / WEIGHT_ONE)
    part = d - torch.log(total.double() / WEIGHT_ONE)
    return (torch.where(none, -1, actions).int(), torch.where(none, -math.inf, full).float(), torch.where(none, -math.inf, part).float())


def _plain_policy(s):
    inv = 1.0 / s["temperature"]
    x = s["logits"].float() * inv
    a, scale, bonus = s["actions"].long()[:, None], s["scale"], s["entropy_coef"]
    d = x - x.amax(1, keepdim=True)
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    p = e / z
    lp = d - torch.log(z)
    entropy = -(p * lp).sum(1)
    chosen = lp.gather(1, a)[:, 0]
    adv = s["advantages"]
    if s["old_log_probs"] is None:
        gain, slope = adv * chosen, adv
    else:
        ratio = torch.exp(chosen - s["old_log_probs"])
        free, held = ratio * adv, ratio.clamp(1 - s["clip"], 1 + s["clip"]) * adv
        gain, slope = torch.minimum(free, held), torch.where(free <= held, free, 0.0)
    loss = -scale * (gain + bonus * entropy)
    grad = p * ((scale * slope)[:, None] + scale * bonus * (lp + entropy[:, None]))
    grad.scatter_add_(1, a, -(scale * slope)[:, None])
    grad *= inv
    live = torch.ones_like(chosen, dtype=torch.bool) if s["mask"] is None else s["mask"]
    return (torch.where(live, loss, 0.0), torch.where(live, chosen, 0.0), torch.where(live, entropy, 0.0),
            torch.where(live[:, None], grad, 0.0).to(s["logits"].dtype))


def _rows_of(cache, table, lens, L):
    """[n, L, Hk, D] cached rows as float32, zero from each length on, and which are there."""
    page = cache.shape[1]
    j = torch.arange(L, device=cache.device)
    there = j[None, :] < lens[:, None]
    ids = table[:, j // page].long() * there
    return torch.where(there[:, :, None, None], cache[ids, (j % page)[None, :]].float(), 0.0), there


def _plain_attend(s):
    q = s["q"].float()
    B, H, D = q.shape
    Hk = s["k"].shape[2]
    r, Lp, Ls, m = H // Hk, s["max_prefix"], s["max_len"], s["most"]
    off = s["group_offsets"].long()
    Gn = off.numel() - 1
    row = torch.arange(B, device=q.device)
    group = torch.searchsorted(off[1:], row, right=True)
    place = row - off[group]
    kp, in_p = _rows_of(s["k"], s["prefix_table"], s["prefix_lens"], Lp)
    vp, _ = _rows_of(s["v"], s["prefix_table"], s["prefix_lens"], Lp)
    ks, in_s = _rows_of(s["k"], s["block_table"], s["lens"], Ls)
    vs, _ = _rows_of(s["v"], s["block_table"], s["lens"], Ls)
    # a group's queries side by side, so that its prompt is multiplied once
    qg = torch.zeros(Gn, m, H, D, device=q.device)
    qg[group, place] = q
    qg = qg.view(Gn, m, Hk, r, D).permute(0, 2, 1, 3, 4).reshape(Gn, Hk, m * r, D)
    sp = (qg @ kp.permute(0, 2, 3, 1)).view(Gn, Hk, m, r, Lp)[group, :, place]                 # [B, Hk, r, Lp]
    ss = q.view(B, Hk, r, D) @ ks.permute(0, 2, 3, 1)
    c = torch.cat([torch.where(in_p[group][:, None, None], sp * s["scale"], -math.inf),
                   torch.where(in_s[:, None, None], ss * s["scale"], -math.inf)], 3)
    top = c.amax(3, keepdim=True)
    e = torch.exp(c - torch.where(top == -math.inf, 0.0, top))
    z = e.sum(3, keepdim=True)
    eg = torch.zeros(Gn, m, Hk, r, Lp, device=q.device)
    eg[group, place] = e[..., :Lp]
    og = eg.permute(0, 2, 1, 3, 4).reshape(Gn, Hk, m * r, Lp) @ vp.permute(0, 2, 1, 3)
    o = og.view(Gn, Hk, m, r, D)[group, :, place] + e[..., Lp:] @ vs.permute(0, 2, 1, 3)
    o = torch.where(z > 0, o / z, 0.0)
    return o.reshape(B, H, D).to(s["q"].dtype), (top + torch.log(z)).reshape(B, H)


def _plain_tables(s):
    page, table, free = s["page"], s["table"], s["free"]
    dev, width = table.device, table.shape[1]
    before, after = s["cached"].long(), s["cached"].long() + s["added"].long()
    have, need = (before + page - 1) // page, (after + page - 1) // page
    first = torch.cumsum(need - have, 0) - (need - have)
    j = torch.arange(width, device=dev)[None, :]
    fresh = (first - have)[:, None] + j
    new = torch.where(j < have[:, None], table, torch.where(j < need[:, None], free[fresh.clamp(0, free.numel() - 1)], -1))
    ends = torch.cumsum(s["added"].long(), 0)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), ends])
    token = torch.arange(s["slots"], device=dev)
    row = torch.searchsorted(ends, token, right=True)
    at = before[row] + token - offsets[row]
    slots = new[row, at // page].long() * page + at % page
    return slots, at.int(), offsets.int(), (need - have).sum().int().reshape(1), new


def run(state):
    s = state
    if not own:
        return {"sample": _plain_sample, "policy": _plain_policy, "attend": _plain_attend, "tables": _plain_tables}[s["op"]](s)
    from paper_2608_17641_b200 import api
    if s["op"] == "sample":
        return api.sample_actions(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    if s["op"] == "policy":
        return api.compute_policy_gradient(s["logits"], s["actions"], s["advantages"], old_log_probs=s["old_log_probs"], mask=s["mask"],
                                           temperature=s["temperature"], clip=s["clip"], entropy_coef=s["entropy_coef"], scale=s["scale"])
    if s["op"] == "attend":
        return api.shared_prefix_attention(s["q"], s["k"], s["v"], s["prefix_table"], s["prefix_lens"], s["group_offsets"], s["block_table"],
                                           s["lens"], scale=s["scale"], max_prefix_len=s["max_prefix"], max_len=s["max_len"])
    return (*api.build_block_tables(s["cached"], s["added"], s["free"], s["table"], page_size=s["page"], num_slots=s["slots"]), s["table"])


# ------------------------------------------------------------------------------------------ work
def work(case):
    """Bytes and operations a pass cannot do without; ragged lengths count with their mean."""
    op = case["op"]
    if op in ("sample", "policy"):
        R, A, size = case["rows"], case["actions"], {"f32": 4, "bf16": 2}[case["dtype"]]
        if op == "sample":
            given = {"none": 4, "both": 16, "mixed": 20}[case["filters"]]
            return {"bytes": R * (A * size + given + 12), "flops": 4 * R * A}
        live = 0.85 if case["padding"] else 1.0
        return {"bytes": R * (A * size * (1 + live) + 8 + (4 if case["clipped"] else 0) + (1 if case["padding"] else 0) + 12),
                "flops": 10 * R * A * live}
    if op == "attend":
        Gn, B, H, Hk, D, page = (case[k] for k in ("groups", "rows", "heads", "kv_heads", "dim", "page"))
        shared, mine = case["prefix"] + (Gn - 1) * 0.75 * case["prefix"], case["own"] + (B - 1) * 0.5 * case["own"]
        mean = shared / Gn
        return {"bytes": (shared + mine) * Hk * D * 4 + B * H * (D * 4 + 4) + 4 * (shared + mine) / page + 8 * (Gn + B),
                "flops": 4 * H * D * (B * mean + mine)}
    B = case["rows"]
    added = B if case["added"] == 1 else B * 0.5 * case["added"]
    width = -(-(case["cached"] + case["added"]) // case["page"])
    return {"bytes": 8 * B + 4 * B * width + 12 * added + 4 * B + 4 * added / case["page"], "flops": B * width + 4 * added}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "tables":
        return None                                       # whole numbers only
    if s["op"] == "sample":
        return _exact_sample(s)
    if s["op"] == "policy":
        return _exact_policy(s)
    return _exact_attend(s)


def _exact_sample(s):
    R, A = s["logits"].shape
    full, part = [], []
    step = max(1, (1 << 26) // A)
    for k in range(0, R, step):
        x = s["logits"][k:k + step].double()
        n = x.shape[0]

        def of(name, other):
            return torch.full((n, 1), other, dtype=torch.float64, device=x.device) if s[name] is None else s[name][k:k + n, None].double()

        t, top_k, top_p, min_p, u = of("temperature", 1.0), of("top_k", 0), of("top_p", 1.0), of("min_p", 0.0), s["uniforms"][k:k + n, None].double()
        y, index = torch.sort(x, dim=1, descending=True, stable=True)
        y = (y - y[:, :1]) / torch.where(t > 0, t, 1.0)
        e = torch.exp(y)                                  # NaN throughout in a row that allows nothing
        rank = torch.arange(A, device=x.device)[None, :]
        bound = torch.where(t > 0, torch.where(top_k > 0, top_k, A), 1)
        alive = (rank < bound) & ((e >= min_p) | (rank == 0))
        f = e * alive
        alive &= (torch.cumsum(f, 1) - f < top_p * f.sum(1, keepdim=True)) | (top_p >= 1) | (rank == 0)
        f = e * alive
        natural = torch.zeros_like(f).scatter_(1, index, f)
        back = torch.zeros_like(f).scatter_(1, index, y)
        run_ = torch.cumsum(natural, 1)
        hit = torch.argmax((run_ > u * run_[:, -1:]).to(torch.uint8), 1, keepdim=True)
        d = back.gather(1, hit)
        empty = x.amax(1, keepdim=True) == -math.inf
        full.append(torch.where(empty, -math.inf, d - torch.log(e.sum(1, keepdim=True)))[:, 0])
        part.append(torch.where(empty, -math.inf, d - torch.log(f.sum(1, keepdim=True)))[:, 0])
    return None, torch.cat(full), torch.cat(part)


def _exact_policy(s):
    R, A = s["logits"].shape
    out = [], [], [], []
    step = max(1, (1 << 26) // A)
    for k in range(0, R, step):
        x = s["logits"][k:k + step].double() / s["temperature"]
        n = x.shape[0]
        lp = torch.log_softmax(x, 1)
        p = torch.exp(lp)
        h = -(p * lp).sum(1, keepdim=True)
        pick = torch.zeros_like(p).scatter_(1, s["actions"][k:k + n, None].long(), 1.0)
        c = (lp * pick).sum(1, keepdim=True)
        adv = s["advantages"][k:k + n, None].double()
        if s["old_log_probs"] is None:
            value, dc = adv * c, adv
        else:
            r = torch.exp(c - s["old_log_probs"][k:k + n, None].double())
            inside = torch.where(adv > 0, r <= 1 + s["clip"], r >= 1 - s["clip"])
            value = torch.where(inside, r, torch.where(adv > 0, 1 + s["clip"], 1 - s["clip"])) * adv
            dc = torch.where(inside, r * adv, 0.0)
        live = torch.ones_like(c) if s["mask"] is None else s["mask"][k:k + n, None].double()
        w = -s["scale"] * live
        out[0].append((w * (value + s["entropy_coef"] * h))[:, 0])
        out[1].append((live * c)[:, 0])
        out[2].append((live * h)[:, 0])
        out[3].append(w * (dc * (pick - p) - s["entropy_coef"] * p * (lp + h)) / s["temperature"])
    return tuple(torch.cat(v) for v in out)


def _exact_attend(s):
    B, H, D = s["q"].shape
    Hk, page = s["k"].shape[2], s["k"].shape[1]
    off = s["group_offsets"].tolist()
    pre, mine = s["prefix_lens"].tolist(), s["lens"].tolist()
    out = torch.zeros(B, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device=DEV)

    def take(cache, table, n):
        return cache[table[:-(-n // page)].long()].reshape(-1, Hk, D)[:n]

    for g in range(len(off) - 1):
        kp, vp = take(s["k"], s["prefix_table"][g], pre[g]), take(s["v"], s["prefix_table"][g], pre[g])
        for b in range(off[g], off[g + 1]):
            k = torch.cat([kp, take(s["k"], s["block_table"][b], mine[b])]).double().repeat_interleave(H // Hk, 1)
            v = torch.cat([vp, take(s["v"], s["block_table"][b], mine[b])]).double().repeat_interleave(H // Hk, 1)
            if not k.shape[0]:
                continue
            c = torch.einsum("hd,lhd->hl", s["q"][b].double(), k) * s["scale"]
            lse[b] = torch.logsumexp(c, 1)
            out[b] = torch.einsum("hl,lhd->hd", torch.softmax(c, 1), v)
    return out, lse
