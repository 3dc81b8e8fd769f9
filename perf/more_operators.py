"""Cases, plain forms and 64-bit definitions of the operators of speculative rollouts and of distillation.

A draft policy proposes tokens, the target policy scores them in one chunk, some are kept, the cache follows, and the draft
policy learns from the target's strongest logits:

  attend   attention of chunks of new tokens (whole prompts, parts of prompts, drafts, single tokens) over a paged cache
  verify   drafted tokens kept or turned down against the target's probabilities, and the token that follows the kept ones
  distill  loss towards the strongest logits of a teacher, and its gradient
  fork     trajectories continued from others: page tables that share whole pages, and copies of the last, part-filled ones
  free     the pages that no trajectory names

``run`` computes the plain form with elementary torch operations where ``own`` is false, and calls the package's operators
where it is true.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WEIGHT_ONE = 2.0 ** 31          # weight of the most likely token: exp(0) in units of 2^-31
SHARE_ONE = 2.0 ** 40           # a probability of 1 where two distributions are subtracted


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one trajectory takes its next token right after a short prompt: latency
        {"name": "attend one token", "op": "attend", "seqs": 1, "new": 1, "cached": 100, "heads": 8, "kv_heads": 8, "dim": 64, "page": 16},
        # a batch of trajectories scores its drafts, one to eight tokens each
        {"name": "attend drafts", "op": "attend", "seqs": 64, "new": 8, "cached": 4096, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64},
        # a new batch of prompts of all lengths, nothing cached
        {"name": "attend prompts", "op": "attend", "seqs": 7, "new": 4096, "cached": 0, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64},
        # part of a long prompt; seven heads on each key head
        {"name": "attend part of a long prompt", "op": "attend", "seqs": 1, "new": 1000, "cached": 32768, "heads": 28, "kv_heads": 4, "dim": 128,
         "page": 128},
        # one trajectory waits for the verdict on its drafts: latency
        {"name": "verify one trajectory", "op": "verify", "seqs": 1, "drafts": 5, "ragged": False, "actions": 131072, "dtype": "bf16", "pad": 0,
         "drawn": True, "temperature": "one", "masked": False},
        # a batch whose trajectories have different numbers of drafts and different temperatures, some of them greedy
        {"name": "verify a batch", "op": "verify", "seqs": 128, "drafts": 7, "ragged": True, "actions": 131072, "dtype": "bf16", "pad": 0,
         "drawn": True, "temperature": "mixed", "masked": False},
        # the draft policy's minibatch of tokens
        {"name": "distill large set", "op": "distill", "rows": 4096, "actions": 131072, "top": 64, "dtype": "bf16", "pad": 0, "padding": False},
        # odd width, padding tokens between the trajectories, float32
        {"name": "distill padded odd rows", "op": "distill", "rows": 1021, "actions": 50021, "top": 20, "dtype": "f32", "pad": 11, "padding": True},
        # a few trajectories branch: latency
        {"name": "fork a few", "op": "fork", "rows": 8, "len": 1000, "page": 16, "kv_heads": 8, "dim": 64},
        # a population of trajectories is resampled
        {"name": "fork a population", "op": "fork", "rows": 2048, "len": 256, "page": 64, "kv_heads": 8, "dim": 128},
        # every step of a rollout: drafts were turned down, some trajectories ended
        {"name": "free a batch", "op": "free", "rows": 128, "len": 4096, "page": 64, "spare": 1000},
        # a large cache of small pages
        {"name": "free a large cache", "op": "free", "rows": 4096, "len": 8192, "page": 16, "spare": 100003},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "verify", "distill", "fork", "free"])
    if op == "attend":
        heads, kv_heads = rng.choice([(8, 8), (16, 2), (32, 8), (28, 4), (20, 1), (32, 32)])
        while True:
            case = {"op": op, "seqs": _log_int(rng, 1, 64), "new": _log_int(rng, 1, 4096), "cached": rng.choice([0, _log_int(rng, 1, 32768)]),
                    "heads": heads, "kv_heads": kv_heads, "dim": rng.choice([64, 128]), "page": rng.choice([16, 32, 64, 128])}
            w = work(case)
            square = case["seqs"] * case["new"] * (case["cached"] + case["new"]) * heads
            if w["flops"] <= 3.0e11 and w["bytes"] <= 8.0e8 and square <= 3 << 30:
                return case
    if op == "verify":
        actions = _log_int(rng, 2, 262144)
        drafts = rng.choice([0, 1, 2, 3, 5, 8, 16])
        return {"op": op, "seqs": _log_int(rng, 1, min(1024, max(1, (1 << 26) // (actions * (drafts + 1))))), "drafts": drafts, "ragged": rng.random() < 0.6,
                "actions": actions, "dtype": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 1, 8, 13]), "drawn": rng.random() < 0.7,
                "temperature": rng.choice(["one", "mixed"]), "masked": rng.random() < 0.3}
    if op == "distill":
        actions = _log_int(rng, 2, 262144)
        return {"op": op, "rows": _log_int(rng, 1, min(262144, (1 << 27) // actions)), "actions": actions, "top": _log_int(rng, 1, min(128, actions)),
                "dtype": rng.choice(["f32", "bf16"]), "pad": rng.choice([0, 0, 1, 8, 13]), "padding": rng.random() < 0.5}
    page, length = rng.choice([16, 32, 64, 100]), _log_int(rng, 1, 4096)
    if op == "fork":
        kv_heads, dim = rng.choice([(8, 64), (2, 128), (8, 128), (1, 64)])
        most = (1 << 28) // (kv_heads * dim * (length + page))
        return {"op": op, "rows": _log_int(rng, 1, max(1, min(2048, most))), "len": length, "page": page, "kv_heads": kv_heads, "dim": dim}
    return {"op": op, "rows": _log_int(rng, 1, 4096), "len": length, "page": page, "spare": _log_int(rng, 1, 100000)}


# ------------------------------------------------------------------------------------------ inputs
def _logits(rows, actions, dtype, pad, g):
    """Rows as a trained policy gives them: a broad bulk and a few strong candidates; `pad` more columns in memory."""
    x = torch.empty(rows, actions + pad, dtype=dtype, device=DEV).normal_(0.0, 2.0, generator=g)
    strong = torch.randint(0, actions, (rows, min(actions, 24)), generator=g, device=DEV)
    x.scatter_reduce_(1, strong, (torch.rand(strong.shape, generator=g, device=DEV) * 8 + 6).to(dtype), "amax")
    return x[:, :actions]


def _chunk_rows(actions):
    return max(1, (1 << 25) // actions)


def _counts(most, n, g):
    """n numbers from 1 to `most`, in pairs that add up to most + 1 (their sum is the same for every seed), shuffled."""
    half = torch.randint(1, most + 1, (n // 2,), generator=g, device=DEV)
    some = torch.cat([half, most + 1 - half, torch.full((n % 2,), (most + 1) // 2 if n > 1 else most, device=DEV)])
    return some[torch.randperm(n, generator=g, device=DEV)]


def _offsets(counts):
    return torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(counts, 0)]).to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    op = case["op"]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    def ints(lo, hi, shape):
        return torch.randint(lo, hi, shape, generator=g, device=DEV, dtype=torch.int32)

    if op == "attend":
        B, H, Hk, D, page = (case[k] for k in ("seqs", "heads", "kv_heads", "dim", "page"))
        counts = _counts(case["new"], B, g)
        T = int(counts.sum())
        cached = ints(case["cached"] // 2, case["cached"] + 1, (B,))
        cached[-1] = case["cached"]
        width = -(-(case["cached"] + case["new"]) // page)
        pages = B * width + 3
        kv = torch.empty(2, pages, page, Hk, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        return {"op": op, "q": torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV).normal_(generator=g), "k": kv[0], "v": kv[1],
                "table": torch.randperm(pages, generator=g, device=DEV)[:B * width].to(torch.int32).view(B, width),
                "offsets": _offsets(counts), "lens": cached + counts.to(torch.int32), "scale": 1.0 / math.sqrt(D),
                "max_new": case["new"], "max_len": case["cached"] + case["new"]}
    if op == "verify":
        B, A, dt = case["seqs"], case["actions"], DTYPES[case["dtype"]]
        counts = _counts(case["drafts"] + 1, B, g) if case["ragged"] else torch.full((B,), case["drafts"] + 1, device=DEV)
        T = int(counts.sum())
        x = _logits(T, A, dt, case["pad"], g)
        t = torch.ones(B, device=DEV)
        if case["temperature"] == "mixed":       # a fifth of the trajectories greedy
            t = torch.where(rand(B) < 0.2, 0.0, rand(B) * 1.2 + 0.3)
        offsets = _offsets(counts)
        if case["masked"]:                       # some tokens are not allowed, and some rows allow none
            x[rand(T, A) < 0.3] = -math.inf
            x[::16] = -math.inf
        drafts = None
        if case["drawn"]:                        # the draft policy is close to the target
            drafts = torch.empty(T, A + case["pad"], dtype=dt, device=DEV)[:, :A]
        tokens = ints(0, A, (T,))
        row_t = torch.repeat_interleave(t, counts)
        for k in range(0, T, _chunk_rows(A)):
            f = x[k:k + _chunk_rows(A)].float() + 0.5 * torch.randn(x[k:k + _chunk_rows(A)].shape, generator=g, device=DEV)
            f = torch.where(f == -math.inf, -20.0, f)
            if drafts is not None:
                drafts[k:k + f.shape[0]] = f.to(dt)
                f = drafts[k:k + f.shape[0]].float()
            noise = -torch.log(-torch.log(torch.rand(f.shape, generator=g, device=DEV).clamp(1e-7, 1 - 1e-6)))
            pick = (f + noise * row_t[k:k + f.shape[0], None]).argmax(1).to(torch.int32)
            tokens[k + 1:k + 1 + f.shape[0]] = pick[:T - 1 - k]
        return {"op": op, "logits": x, "draft_logits": drafts, "tokens": tokens, "offsets": offsets, "uniforms": rand(T), "draw_uniforms": rand(B),
                "temperature": t if case["temperature"] == "mixed" else None}
    if op == "distill":
        R, A, k = case["rows"], case["actions"], case["top"]
        x = _logits(R, A, DTYPES[case["dtype"]], case["pad"], g)
        ids, top = torch.empty(R, k, dtype=torch.int32, device=DEV), torch.empty(R, k, device=DEV)
        for at in range(0, R, _chunk_rows(A)):   # the teacher agrees with the student about most of the strong candidates
            f = x[at:at + _chunk_rows(A)].float()
            v, i = torch.topk(f + torch.randn(f.shape, generator=g, device=DEV), k, dim=1)
            top[at:at + f.shape[0]], ids[at:at + f.shape[0]] = v, i.to(torch.int32)
        s = {"op": op, "logits": x, "ids": ids, "teacher": top, "mask": None, "temperature": 1.5, "scale": 1.5 ** 2 / R}
        if case["padding"]:                      # padding tokens, and teachers that give fewer candidates
            s["mask"] = rand(R) < 0.85
            ids[torch.arange(k, device=DEV)[None, :] >= ints(max(1, k // 2), k + 1, (R, 1))] = -1
        return s
    rows, page = case["rows"], case["page"]
    lens = ints(case["len"] // 2, case["len"] + 1, (rows,))
    lens[0] = case["len"]
    width = -(-case["len"] // page)
    have = (lens + page - 1) // page
    if op == "fork":
        held = int(have.sum())
        pages = rows * width + rows
        ids = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(width, device=DEV)[None, :] < have[:, None]] = ids[:held]
        kv = torch.empty(2, pages, page, case["kv_heads"], case["dim"], dtype=torch.bfloat16, device=DEV).normal_(generator=g)
        return {"op": op, "table": table, "lens": lens, "sources": ints(0, rows, (rows,)), "free": ids[held:held + rows], "k": kv[0], "v": kv[1],
                "page": page}
    pages = rows * width + case["spare"]
    table = torch.randperm(pages, generator=g, device=DEV)[:rows * width].to(torch.int32).view(rows, width)
    some = rand(rows)
    table[: rows // 4, : width // 2] = table[rows - rows // 4:, : width // 2]        # branches of a common beginning
    return {"op": op, "table": table, "lens": torch.where(some < 0.1, 0, lens), "page": page, "pages": pages}


# ------------------------------------------------------------------------------------------ plain forms
def _plain_attend(s):
    q, page = s["q"].float(), s["k"].shape[1]
    T, H, D = q.shape
    Hk, dev = s["k"].shape[2], q.device
    r, N, L = H // Hk, s["max_new"], s["max_len"]
    off, lens = s["offsets"].long(), s["lens"].long()
    B = lens.numel()
    counts = off[1:] - off[:-1]
    token = torch.arange(T, device=dev)
    seq = torch.searchsorted(off[1:], token, right=True)
    place = token - off[seq]
    j = torch.arange(L, device=dev)
    there = j[None, :] < lens[:, None]
    ids = s["table"][:, j // page].long() * there
    i = torch.arange(N, device=dev)
    sees = j[None, None, :] <= ((lens - counts)[:, None] + i[None, :])[:, :, None]                   # [B, N, L]
    out, lse = torch.empty(T, H, D, device=dev), torch.empty(T, H, device=dev)
    for h in range(Hk):
        k = torch.where(there[:, :, None], s["k"][ids, (j % page)[None, :], h].float(), 0.0)           # [B, L, D]
        v = torch.where(there[:, :, None], s["v"][ids, (j % page)[None, :], h].float(), 0.0)
        qh = torch.zeros(B, N, r, D, device=dev)
        qh[seq, place] = q[:, h * r:(h + 1) * r]
        c = (qh.view(B, N * r, D) @ k.transpose(1, 2)).view(B, N, r, L) * s["scale"]
        c.masked_fill_(~sees[:, :, None, :], -math.inf)
        top = c.amax(3, keepdim=True)
        c -= torch.where(top == -math.inf, 0.0, top)
        e = c.exp_()
        z = e.sum(3, keepdim=True)
        o = (e.view(B, N * r, L) @ v).view(B, N, r, D)
        o = torch.where(z > 0, o / z, 0.0)
        out[:, h * r:(h + 1) * r] = o[seq, place]
        lse[:, h * r:(h + 1) * r] = (top + torch.log(z))[seq, place, :, 0]
    return out.to(s["q"].dtype), lse


def _plain_weights(x, inv):
    """Distance to the row's maximum, sum of its exponentials and whole weights 2^31 exp; nothing where a row allows nothing."""
    top = x.amax(1, keepdim=True)
    d = torch.where(x == top, 0.0, (x - top) * inv[:, None])
    e = torch.where(top == -math.inf, 0.0, torch.exp(d))
    return d, e.sum(1, dtype=torch.float64), torch.floor(e.double() * WEIGHT_ONE + 0.5).long()


def _plain_verify(s):
    x, dev = s["logits"], s["logits"].device
    T, A = x.shape
    off = s["offsets"].long()
    B = off.numel() - 1
    row = torch.arange(T, device=dev)
    seq = torch.searchsorted(off[1:], row, right=True)
    last = row == off[seq + 1] - 1
    t = torch.ones(B, device=dev) if s["temperature"] is None else s["temperature"]
    greedy = ~(t > 0)
    inv = 1.0 / torch.where(greedy, 1.0, t)
    drafted = torch.where(last, -1, torch.cat([s["tokens"][1:].long(), s["tokens"].new_zeros(1).long()]))
    at = drafted.clamp(0, A - 1)[:, None]
    valid = (drafted >= 0) & (drafted < A)
    wx, W, vx, V, dx, S = (torch.zeros(T, dtype=torch.float64, device=dev) for _ in range(6))
    step = max(1, (1 << 27) // A)
    for k in range(0, T, step):
        f, i = x[k:k + step].float(), inv[seq[k:k + step]]
        d, sums, w = _plain_weights(f, i)
        best = torch.argmax(f, 1)                                                                    # the first of equals
        one = torch.zeros_like(w).scatter_(1, best[:, None], 1) * (sums > 0)[:, None]
        w = torch.where(greedy[seq[k:k + step], None], one, w)
        here = at[k:k + step]
        wx[k:k + step], W[k:k + step], S[k:k + step] = w.gather(1, here)[:, 0].double(), w.sum(1).double(), sums
        dx[k:k + step] = d.gather(1, here)[:, 0].double()
        if s["draft_logits"] is not None:
            _, _, v = _plain_weights(s["draft_logits"][k:k + step].float(), i)
            vx[k:k + step], V[k:k + step] = v.gather(1, here)[:, 0].double(), v.sum(1).double()
    if s["draft_logits"] is None:
        vx += 1
        V += 1
    u = s["uniforms"].double()
    keep = valid & ~last & torch.where(greedy[seq], wx > 0, u * (vx * W) < wx * V)
    # the first row of each trajectory whose draft is not kept
    stop = torch.full((B,), T, dtype=torch.long, device=dev).scatter_reduce_(0, seq, torch.where(keep, T, row), "amin")
    tokens = torch.where(row < stop[seq], drafted, -1)
    log_probs = torch.where(row < stop[seq], dx - torch.log(S), -math.inf)
    there = off[1:] > off[:-1]
    stop = torch.where(there, stop, 0)
    for k in range(0, B, step):                                                                      # the token after the kept ones
        r = stop[k:k + step]
        f, g = x[r].float(), greedy[k:k + step]
        i = inv[k:k + step]
        d, sums, w = _plain_weights(f, i)
        best = torch.argmax(f, 1)
        w = torch.where(g[:, None], torch.zeros_like(w).scatter_(1, best[:, None], 1), w)
        rest = w
        turned = ~last[r]
        if s["draft_logits"] is not None:
            _, _, v = _plain_weights(s["draft_logits"][r].float(), i)
            share = torch.floor(w.double() * (SHARE_ONE / w.sum(1, keepdim=True).double())).long()
            less = torch.floor(v.double() * (SHARE_ONE / v.sum(1, keepdim=True).double())).long()
            rest = (share - torch.where(v.sum(1, keepdim=True) > 0, less, 0)).clamp(min=0)
        else:
            rest = torch.where(torch.arange(A, device=dev)[None, :] == drafted[r][:, None], 0, w)
        plain = g | ~turned | (rest.sum(1) == 0)
        rest = torch.where(plain[:, None], w, rest)
        total = rest.sum(1)
        target = torch.minimum(torch.floor(s["draw_uniforms"][k:k + step].double() * total.double()).long(), total - 1)
        pick = (torch.cumsum(rest, 1) <= target[:, None]).sum(1).clamp(max=A - 1)
        none = sums == 0
        tokens[r] = torch.where(there[k:k + step], torch.where(none, -1, pick), tokens[r])
        lp = d.gather(1, pick[:, None])[:, 0].double() - torch.log(sums)
        log_probs[r] = torch.where(there[k:k + step], torch.where(none, -math.inf, lp), log_probs[r])
    accepted = torch.where(there, stop - off[:-1], 0)
    return tokens.int(), log_probs.float(), accepted.int()


def _plain_distill(s):
    inv, scale = 1.0 / s["temperature"], s["scale"]
    x = s["logits"].float() * inv
    A = x.shape[1]
    d = x - x.amax(1, keepdim=True)
    q = torch.exp(d)
    z = q.sum(1, keepdim=True)
    q /= z
    ids = s["ids"].long()
    valid = (ids >= 0) & (ids < A)
    at = torch.where(valid, ids, 0)
    t = torch.where(valid, s["teacher"] * inv, -math.inf)
    t = t - t.amax(1, keepdim=True)
    e = torch.exp(t)
    total = e.sum(1, keepdim=True)
    p = e / total
    some = p > 0
    loss = scale * torch.where(some, p * (t - torch.log(total) - d.gather(1, at) + torch.log(z)), 0.0).sum(1)
    q.scatter_add_(1, at, torch.where(some, -p, 0.0))
    q *= scale * inv
    live = valid.any(1)
    if s["mask"] is not None:
        live &= s["mask"]
    return torch.where(live, loss, 0.0), torch.where(live[:, None], q, 0.0).to(s["logits"].dtype)


def _plain_fork(s):
    page, table, src = s["page"], s["table"], s["sources"].long()
    dev, width = table.device, table.shape[1]
    n = src.numel()
    i = torch.arange(n, device=dev)
    length = s["lens"][src].long()
    have = (length + page - 1) // page
    first = torch.full((table.shape[0],), n, dtype=torch.long, device=dev).scatter_reduce_(0, src, i, "amin")[src] == i
    end = (have - 1).clamp(min=0)
    new = torch.where(torch.arange(width, device=dev)[None, :] < have[:, None], table[src], -1)
    old = new.gather(1, end[:, None])[:, 0]
    fresh = ~first & (length % page != 0) & (old >= 0)
    number = torch.cumsum(fresh.long(), 0) - fresh.long()
    page_of = s["free"][number.clamp(max=s["free"].numel() - 1)]
    new.scatter_(1, end[:, None], torch.where(fresh, page_of, old)[:, None])
    come, go = torch.where(fresh, old, -1), torch.where(fresh, page_of, -1)
    # rows that copy nothing copy a page of the table onto itself
    any_page = table[0, 0]
    a, b = torch.where(fresh, come, any_page).long(), torch.where(fresh, go, any_page).long()
    for cache in (s["k"], s["v"]):
        cache[b] = cache[a]
    return new, come, go, fresh.sum().int().reshape(1), s["k"], s["v"]


def _plain_free(s):
    page, table, n = s["page"], s["table"], s["pages"]
    dev = table.device
    live = torch.arange(table.shape[1], device=dev)[None, :] * page < s["lens"][:, None]
    used = torch.zeros(n + 1, dtype=torch.bool, device=dev)
    used[torch.where(live, table, n).long().reshape(-1)] = True
    spare = ~used[:n]
    at = torch.cumsum(spare.long(), 0) - 1
    out = torch.full((n + 1,), -1, dtype=torch.int32, device=dev)
    out.scatter_(0, torch.where(spare, at, n), torch.arange(n, dtype=torch.int32, device=dev))
    return out[:n], spare.sum().int().reshape(1)


def run(state):
    s = state
    if not own:
        return {"attend": _plain_attend, "verify": _plain_verify, "distill": _plain_distill, "fork": _plain_fork, "free": _plain_free}[s["op"]](s)
    from paper_2608_17641_b200 import api
    if s["op"] == "attend":
        return api.chunk_attention(s["q"], s["k"], s["v"], s["table"], s["offsets"], s["lens"], scale=s["scale"], max_new=s["max_new"],
                                   max_len=s["max_len"])
    if s["op"] == "verify":
        return api.verify_drafts(s["logits"], s["tokens"], s["offsets"], s["uniforms"], s["draw_uniforms"], draft_logits=s["draft_logits"],
                                 temperature=s["temperature"])
    if s["op"] == "distill":
        return api.compute_distillation(s["logits"], s["ids"], s["teacher"], mask=s["mask"], temperature=s["temperature"], scale=s["scale"])
    if s["op"] == "fork":
        table, come, go, used = api.fork_block_tables(s["table"], s["lens"], s["sources"], s["free"], page_size=s["page"])
        api.copy_pages(s["k"], s["v"], come, go)
        return table, come, go, used, s["k"], s["v"]
    return api.list_free_pages(s["table"], s["lens"], num_pages=s["pages"], page_size=s["page"])


# ------------------------------------------------------------------------------------------ work
def work(case):
    """Bytes and operations a pass cannot do without; ragged lengths count with their mean."""
    op = case["op"]
    if op == "attend":
        B, N, L, H, Hk, D, page = (case[k] for k in ("seqs", "new", "cached", "heads", "kv_heads", "dim", "page"))
        old = L + (B - 1) * 0.75 * L
        new = B * (N + 1) / 2 if B > 1 else N
        square = B * (N + 1) * (2 * N + 1) / 6 if B > 1 else N * N                            # sum of the counts' squares
        pairs = old * new / B + square / 2 + new / 2
        return {"bytes": (old + new) * Hk * D * 4 + new * H * (D * 4 + 4) + 4 * (old + new) / page + 8 * B, "flops": 4 * H * D * pairs}
    if op in ("verify", "distill"):
        A, size = case["actions"], {"f32": 4, "bf16": 2}[case["dtype"]]
        if op == "verify":
            B = case["seqs"]
            T = B * (case["drafts"] + 2) / 2 if case["ragged"] else B * (case["drafts"] + 1)
            read = T + (T - B if case["drawn"] else 0)
            return {"bytes": read * A * size + T * 16 + B * 16, "flops": 4 * read * A}
        R = case["rows"]
        live = 0.85 if case["padding"] else 1.0
        return {"bytes": R * (A * size * (1 + live) + 8 * case["top"] * live + 4 + (1 if case["padding"] else 0)), "flops": 8 * R * A * live}
    rows, page = case["rows"], case["page"]
    entries = rows * (0.75 * case["len"] / page + 0.5)
    width = -(-case["len"] // page)
    if op == "fork":
        copies = (rows - rows * (1 - (1 - 1 / rows) ** rows)) * (1 - 1 / page)
        return {"bytes": 4 * (entries + rows * width + 5 * rows) + copies * page * case["kv_heads"] * case["dim"] * 8, "flops": rows * width}
    pages = rows * width + case["spare"]
    return {"bytes": 4 * (0.9 * entries + rows + pages), "flops": entries + pages}


# ------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    if case["op"] in ("fork", "free"):
        return None                                       # whole numbers and copies only
    s = prepare(case, seed)
    return {"attend": _exact_attend, "verify": _exact_verify, "distill": _exact_distill}[case["op"]](s)


def _exact_attend(s):
    T, H, D = s["q"].shape
    page, Hk = s["k"].shape[1], s["k"].shape[2]
    off, lens = s["offsets"].tolist(), s["lens"].tolist()
    out = torch.zeros(T, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        pages = s["table"][b, :-(-n // page)].long()
        k, v = (c[pages].reshape(-1, Hk, D)[:n].double() for c in (s["k"], s["v"]))
        count = off[b + 1] - off[b]
        step = max(1, (1 << 28) // (n * (H // Hk)))
        for i in range(0, count, step):
            m = min(step, count - i)
            rows = slice(off[b] + i, off[b] + i + m)
            later = torch.arange(n, device=DEV)[None, :] > torch.arange(n - count + i, n - count + i + m, device=DEV)[:, None]
            for h in range(Hk):
                heads = slice(h * (H // Hk), (h + 1) * (H // Hk))
                c = torch.einsum("thd,ld->htl", s["q"][rows, heads].double(), k[:, h]) * s["scale"]
                c.masked_fill_(later[None], -math.inf)
                lse[rows, heads] = torch.logsumexp(c, 2).T
                out[rows, heads] = torch.einsum("htl,ld->thd", torch.softmax(c, 2), v[:, h])
    return out, lse


def _exact_verify(s):
    """Log-probabilities of the tokens that the rule gives with real numbers in place of whole weights."""
    off, A = s["offsets"].tolist(), s["logits"].shape[1]
    u, du = s["uniforms"].tolist(), s["draw_uniforms"].tolist()
    tokens, drafts = s["tokens"].tolist(), s["draft_logits"]
    temps = [1.0] * (len(off) - 1) if s["temperature"] is None else s["temperature"].double().tolist()
    out = torch.full((off[-1],), -math.inf, dtype=torch.float64, device=DEV)

    def first_over(weights, share):
        run_ = torch.cumsum(weights, 0)
        return int(torch.argmax((run_ > share * run_[-1]).to(torch.uint8)))

    for b, t in enumerate(temps):
        for r in range(off[b], off[b + 1]):
            x = s["logits"][r].double()
            if x.max() == -math.inf:
                break
            lp = torch.log_softmax(x / t if t > 0 else x, 0)
            p, token, end = lp.exp(), tokens[r + 1] if r + 1 < off[b + 1] else -1, r + 1 == off[b + 1]
            if t <= 0:
                best = int(x.argmax())
                out[r] = lp[best]
                if token != best or end:
                    break
                continue
            q = None if drafts is None else torch.softmax(drafts[r].double() / t, 0)
            if not end and u[r] * (1.0 if q is None else float(q[token])) < float(p[token]):
                out[r] = lp[token]
                continue
            left = p.clone()
            if not end and q is None:
                left[token] = 0.0
            elif not end:
                left = (p - q).clamp(min=0.0)
            out[r] = lp[first_over(left if float(left.sum()) > 0 else p, du[b])]
            break
    return None, out, None


def _exact_distill(s):
    R, A = s["logits"].shape
    losses, grads = [], []
    step = max(1, (1 << 26) // A)
    for k in range(0, R, step):
        lq = torch.log_softmax(s["logits"][k:k + step].double() / s["temperature"], 1)
        ids = s["ids"][k:k + step].long()
        live = (ids >= 0) & (ids < A)
        t = (s["teacher"][k:k + step].double() / s["temperature"]).masked_fill(~live, -math.inf)
        on = live.any(1, keepdim=True) if s["mask"] is None else live.any(1, keepdim=True) & s["mask"][k:k + step, None]
        lp = torch.log_softmax(t, 1)
        p = lp.exp()
        terms = torch.where(p > 0, p * (lp - lq.gather(1, ids.clamp(0, A - 1))), 0.0)
        losses.append(s["scale"] * (terms.sum(1, keepdim=True) * on)[:, 0])
        dense = torch.zeros_like(lq).scatter_add_(1, ids.clamp(0, A - 1), torch.where(live, p, 0.0))
        grads.append(torch.where(on, s["scale"] / s["temperature"] * (lq.exp() - dense), 0.0))
    return torch.cat(losses), torch.cat(grads)
