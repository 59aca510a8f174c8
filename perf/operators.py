"""Measured cases of the operators around a long decode step over the paged KV cache.

Four operators, each in a plain torch form (`own` false) and as the call a user makes of the
library (`own` true):

  rope    KvPool.kv_append_rope: new queries and keys rotated by their positions, keys and values
          written to their pages; one or a few tokens per request, or ragged prompts.
  index   KvPool.kv_index_update (and kv_index_values): 8-bit lower and upper bounds of the keys of
          every page, what page selection scores against.
  sparse  KvPool.decode_attention_sparse: each request's best pages by those bounds, then attention
          of its new token over the chosen pages alone.
  verify  draft_verify: drafted tokens accepted or replaced by the target's probabilities, from
          given random numbers.

Shapes are this repository's workloads' (8B and 70B head layouts, the small one of its tests, the
skewed 131072-token batch) or generic.  `prepare` makes the inputs on the GPU from the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
DEV = "cuda"


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one request of an interactive instance: latency of a single decode token
        dict(name="rope_one_token", op="rope", batch=1, heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False,
             new_lo=1, new_hi=1, ctx_lo=4096, ctx_hi=4096, packed=True),
        # speculative decoding: five new tokens for each request of the 70B-shaped batch, far positions
        dict(name="rope_drafts_b96", op="rope", batch=96, heads=64, kv_heads=8, dim=128, rotary=128, interleaved=False,
             new_lo=5, new_hi=5, ctx_lo=1024, ctx_hi=4096, packed=True),
        # ragged prompts entering the cache, some as continuation chunks, half of each head rotated in pairs
        dict(name="rope_prompts_b8", op="rope", batch=8, heads=32, kv_heads=8, dim=128, rotary=64, interleaved=True,
             new_lo=37, new_hi=8191, ctx_lo=0, ctx_hi=120001, packed=False),
        # a short prompt's pages summarised
        dict(name="index_prompt_333", op="index", batch=1, heads=4, kv_heads=1, dim=64, ctx_lo=333, ctx_hi=333),
        # a batch of long prompts summarised before sparse decoding starts
        dict(name="index_prompts_b8", op="index", batch=8, heads=32, kv_heads=8, dim=128, ctx_lo=4001, ctx_hi=32768),
        # one request with a long context: latency
        dict(name="sparse_one_131072", op="sparse", batch=1, heads=32, kv_heads=8, dim=128, ctx_lo=131072, ctx_hi=131072,
             budget=128, sink=1, recent=2),
        # the small head layout, lengths around and below the budget (some requests are not cut at all)
        dict(name="sparse_small_b5", op="sparse", batch=5, heads=4, kv_heads=1, dim=64, ctx_lo=1, ctx_hi=2999,
             budget=24, sink=1, recent=2),
        # a batch of long-context requests on the 8B shape
        dict(name="sparse_b64", op="sparse", batch=64, heads=32, kv_heads=8, dim=128, ctx_lo=8192, ctx_hi=32768,
             budget=128, sink=1, recent=4),
        # the 70B-shaped batch with a small budget: selection weighs as much as attention
        dict(name="sparse_b96_g8", op="sparse", batch=96, heads=64, kv_heads=8, dim=128, ctx_lo=1024, ctx_hi=16384,
             budget=33, sink=2, recent=2),
        # one request's drafts against a full-size vocabulary: latency
        dict(name="verify_one", op="verify", batch=1, drafts=4, vocab=128256, dtype="float32", draft_probs=True, ragged=False),
        # an interactive batch, ragged numbers of drafts, probabilities in 16 bits, odd vocabulary
        dict(name="verify_b64_bf16", op="verify", batch=64, drafts=7, vocab=50257, dtype="bfloat16", draft_probs=True, ragged=True),
        # a large batch whose drafts come without probabilities (looked up in the prompt, say)
        dict(name="verify_b256_lookup", op="verify", batch=256, drafts=3, vocab=128256, dtype="float32", draft_probs=False, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (64, 8, 128), (8, 2, 128), (4, 1, 64), (12, 4, 64), (6, 6, 128), (35, 5, 128)])
    op = rng.choice(["rope", "index", "sparse", "verify"])
    if op == "verify":
        batch, drafts, vocab = _log_int(rng, 1, 256), rng.randint(1, 8), _log_int(rng, 1000, 151936)
        batch = max(1, min(batch, int(1.3e8 / ((drafts + 1) * vocab))))
        return dict(op=op, batch=batch, drafts=drafts, vocab=vocab, dtype=rng.choice(["float32", "bfloat16"]),
                    draft_probs=rng.random() < 0.7, ragged=rng.random() < 0.5)
    case = dict(op=op, batch=_log_int(rng, 1, 96), heads=heads, kv_heads=kv_heads, dim=dim)
    if op == "rope":
        ragged = rng.random() < 0.5
        most = _log_int(rng, 1, 8191) if ragged else rng.randint(1, 8)
        case["batch"] = max(1, min(case["batch"], int(1400000 * 128 / (most * (heads + 2 * kv_heads) * dim))))
        low = rng.randint(0, most) if ragged else most
        rotary = rng.choice([dim, dim // 2, 16])
        ctx = _log_int(rng, 1, 100000)
        case["batch"] = max(1, min(case["batch"], int(600000 / (ctx + most))))
        case.update(rotary=rotary, interleaved=rng.random() < 0.5, new_lo=low, new_hi=most, ctx_lo=rng.randint(0, ctx), ctx_hi=ctx,
                    packed=rng.random() < 0.5)
        return case
    ctx = _log_int(rng, 1, 131072)
    case["batch"] = max(1, min(case["batch"], int((140000 if op == "index" else 1000000) * 1024 / (ctx * kv_heads * dim))))
    case.update(ctx_lo=rng.randint(1, ctx), ctx_hi=ctx)
    if op == "sparse":
        sink, recent = rng.randint(0, 4), rng.randint(1, 8)
        most = max(4, min(180, int(8000 * 1024 / (case["batch"] * kv_heads * dim))))
        case.update(budget=sink + recent + _log_int(rng, 1, most), sink=sink, recent=recent)
    return case


# ------------------------------------------------------------------------------------ the inputs

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, the same for every seed (what is read depends on their sum)."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _lengths(case):
    """(context lengths after the step, new tokens) of the requests."""
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], case["batch"])
    if case["op"] != "rope":
        return ctx, [0] * len(ctx)
    new = _spread(case["new_lo"], case["new_hi"], case["batch"])[::-1]
    return [c + n for c, n in zip(ctx, new)], new


def _pages(length):
    return (length + PAGE - 1) // PAGE


def _keys(shape, gen):
    """Keys as a model's are: pages with a direction of their own, a few large channels."""
    k = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
    k += 0.7 * torch.randn(shape[:2] + (1,) + shape[3:], generator=gen, device=DEV)
    k[..., ::31] *= 3.0
    return k


def _pool(pages, kv_heads, dim, gen):
    """bf16 [pages][kv_heads][2][16][dim], filled a part at a time."""
    pool = torch.empty(pages, kv_heads, 2, PAGE, dim, dtype=torch.bfloat16, device=DEV)
    for at in range(0, pages, 8192):
        part = pool[at:at + 8192]
        part[:, :, 0] = _keys((part.shape[0], kv_heads, PAGE, dim), gen)
        part[:, :, 1] = torch.randn(part.shape[0], kv_heads, PAGE, dim, generator=gen, device=DEV)
    return pool


def _tables(lens, gen):
    """(block tables, pages of the pool): every request's pages anywhere in the pool."""
    counts = [_pages(n) for n in lens]
    total = sum(counts)
    pages = total + max(1, total // 50)
    order = torch.randperm(pages, generator=gen, device=DEV, dtype=torch.int32)
    tables = torch.full((len(lens), max(1, max(counts))), -1, dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(counts):
        tables[r, :n] = order[at:at + n]
        at += n
    return tables, pages


def _handle(case, state, pages):
    """The library's handle over the pool, as a serving program keeps it."""
    from paper_2501_08090_b200 import binding
    cfg = binding.make_config(1, case["heads"], case["kv_heads"], case["dim"], pages, state["tables"].shape[1], case["batch"])
    return binding.KvPool(cfg, device="cuda:0", pool=state["pool"].view(-1))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"case": case}
    if case["op"] == "verify":
        return _prepare_verify(case, state, gen)
    lens, new = _lengths(case)
    mix = torch.randperm(len(lens), generator=gen, device=DEV).tolist()
    lens, new = [lens[i] for i in mix], [new[i] for i in mix]
    B, H, K, D = case["batch"], case["heads"], case["kv_heads"], case["dim"]
    state["tables"], pages = _tables(lens, gen)
    state["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    state["pool"] = _pool(pages, K, D, gen)
    if case["op"] == "rope":
        T = sum(new)
        if case["packed"]:     # one projection gives queries, keys and values side by side
            qkv = torch.randn(T, H + 2 * K, D, generator=gen, device=DEV).to(torch.bfloat16)
            state["q"], state["k"], state["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        else:
            state["q"], state["k"], state["v"] = (torch.randn(T, h, D, generator=gen, device=DEV).to(torch.bfloat16) for h in (H, K, K))
        half = case["rotary"] // 2
        state["inv_freq"] = (500000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
        state["new_start"] = torch.tensor([0] + new, device=DEV).cumsum(0).to(torch.int32) if min(new) != max(new) else None
        state["q_out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
    else:
        state["index"] = torch.zeros(pages * K * (2 * D + 4), dtype=torch.uint8, device=DEV)
        if case["op"] == "index":
            state["values"] = torch.empty(pages, K, 2, D, dtype=torch.bfloat16, device=DEV)
        else:
            _fill_index(state, pages, K, D)
            q = torch.randn(B, H, D, generator=gen, device=DEV)
            q += 0.7 * torch.randn(B, 1, D, generator=gen, device=DEV)
            state["q"] = q.to(torch.bfloat16)
            state["out"] = torch.empty(B, H, D, dtype=torch.bfloat16, device=DEV)
            state["sel"] = torch.empty(B, K, case["budget"], dtype=torch.int32, device=DEV)
            state["sel_lens"] = torch.empty(B, dtype=torch.int32, device=DEV)
    if own:
        state["handle"] = _handle(case, state, pages)
    return state


def _prepare_verify(case, state, gen):
    B, K, V = case["batch"], case["drafts"], case["vocab"]
    dtype = getattr(torch, case["dtype"])
    target = torch.empty(B, K + 1, V, dtype=dtype, device=DEV)
    draft = torch.empty(B, K, V, dtype=dtype, device=DEV) if case["draft_probs"] else None
    tokens = torch.empty(B, K, dtype=torch.int32, device=DEV)
    for b in range(0, B, 32):
        logits = 2.5 * torch.randn(min(32, B - b), K + 1, V, generator=gen, device=DEV)
        target[b:b + 32] = torch.softmax(logits, -1)
        # a draft model that mostly agrees with the target: tilted logits, tokens sampled from it
        q = torch.softmax(logits[:, :K] + 0.4 * torch.randn(logits.shape[0], K, V, generator=gen, device=DEV), -1)
        if draft is not None:
            draft[b:b + 32] = q
        tokens[b:b + 32] = torch.multinomial(q.view(-1, V), 1, generator=gen).view(-1, K).int()
    state.update(target=target, draft=draft, drafted=tokens, u_accept=torch.rand(B, K, generator=gen, device=DEV),
                 u_sample=torch.rand(B, generator=gen, device=DEV), draft_lens=None)
    if draft is None:      # point masses: a lookup that is right about two times in three
        sure = torch.rand(B, K, generator=gen, device=DEV) < 0.65
        peak = torch.where(sure, 0.9, 0.05).to(dtype)
        at = tokens.long().unsqueeze(-1)
        rows = target[:, :K]
        rows *= (1 - peak).unsqueeze(-1)
        rows.scatter_add_(2, at, peak.unsqueeze(-1))
    if case["ragged"]:
        lens = torch.tensor(_spread(0, K, B), dtype=torch.int32, device=DEV)
        state["draft_lens"] = lens[torch.randperm(B, generator=gen, device=DEV)]
    state["tokens"] = torch.empty(B, K + 1, dtype=torch.int32, device=DEV)
    state["accepted"] = torch.empty(B, dtype=torch.int32, device=DEV)
    return state


# ------------------------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(op, state)
    return {"rope": _rope, "index": _index, "sparse": _sparse, "verify": _verify}[op](state)


def _run_own(op, s):
    from paper_2501_08090_b200 import binding
    case = s["case"]
    if op == "verify":
        binding.draft_verify(s["drafted"], s["target"], s["draft"], s["u_accept"], s["u_sample"], s["tokens"], s["accepted"],
                             draft_lens=s["draft_lens"])
        return {"tokens": s["tokens"], "accepted": s["accepted"]}
    kp = s["handle"]
    if op == "rope":
        kp.kv_append_rope(0, s["tables"], s["lens"], s["q"], s["k"], s["v"], s["q_out"], s["inv_freq"], new_start=s["new_start"],
                          interleaved=case["interleaved"])
        return {"q": s["q_out"], "pool": s["pool"]}
    if op == "index":
        kp.kv_index_update(0, s["tables"], s["lens"], s["index"])
        kp.kv_index_values(0, s["index"], s["values"])
        return {"values": s["values"]}
    kp.decode_attention_sparse(0, s["tables"], s["lens"], s["q"], s["index"], s["sel"], s["sel_lens"], s["out"],
                               sink=case["sink"], recent=case["recent"])
    return {"out": s["out"], "pages": s["sel"], "lens": s["sel_lens"]}


# ---- rope: x' = x cos(a) - y sin(a), y' = y cos(a) + x sin(a), a = position * inv_freq

def _rotate(x, cos, sin, half, interleaved):
    x = x.float()
    a, b, rest = (x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]) if interleaved else \
        (x[..., :half], x[..., half:2 * half], x[..., 2 * half:])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), -1).flatten(-2) if interleaved else torch.cat((ra, rb), -1)
    return torch.cat((turned, rest), -1).to(torch.bfloat16)


def _rope(s):
    T, lens = s["q"].shape[0], s["lens"].long()
    if s["new_start"] is None:
        each = T // lens.numel()
        starts = torch.arange(lens.numel() + 1, device=DEV) * each
    else:
        starts = s["new_start"].long()
    i = torch.arange(T, device=DEV)
    r = torch.searchsorted(starts, i, right=True) - 1
    pos = lens[r] - (starts[r + 1] - starts[r]) + (i - starts[r])
    angle = pos.double().unsqueeze(-1) * s["inv_freq"].double()
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    half, inter = s["inv_freq"].numel(), s["case"]["interleaved"]
    page, slot = s["tables"][r, pos // PAGE].long(), pos % PAGE
    s["pool"][page, :, 0, slot] = _rotate(s["k"], cos, sin, half, inter)
    s["pool"][page, :, 1, slot] = s["v"]
    return {"q": _rotate(s["q"], cos, sin, half, inter), "pool": s["pool"]}


# ---- index: lo <= k <= hi over a page's keys, in whole steps of a power of two per (page, head)

def _two_to(exp):
    """2^exp as fp32, for whole exponents of normal numbers (a power function may be off by a rounding)."""
    return ((exp.int() + 127) << 23).view(torch.float32)


def _bounds(keys, valid):
    """(lo, hi int8 [..., d], step fp32 [...]) of keys [..., 16, d] whose slots `valid` [..., 16] count."""
    keys = keys.float()
    low = keys.masked_fill(~valid.unsqueeze(-1), math.inf).amin(-2)
    high = keys.masked_fill(~valid.unsqueeze(-1), -math.inf).amax(-2)
    most = torch.maximum(low.abs(), high.abs()).amax(-1)
    exp = torch.frexp(most.clamp_min(2.0 ** -100))[1] - 7
    exp = torch.where(torch.ceil(most / _two_to(exp)) > 127, exp + 1, exp)
    step = _two_to(exp)
    lo, hi = torch.floor(low / step.unsqueeze(-1)), torch.ceil(high / step.unsqueeze(-1))
    return lo.to(torch.int8), hi.to(torch.int8), step


def _index_views(index, pages, kv_heads, dim):
    cut = pages * kv_heads * 2 * dim
    return index[:cut].view(torch.int8).view(pages, kv_heads, 2, dim), index[cut:].view(torch.float32).view(pages, kv_heads)


def _fill_index(s, pages, kv_heads, dim):
    rec, step = _index_views(s["index"], pages, kv_heads, dim)
    n = (s["lens"].long() + PAGE - 1) // PAGE
    col = torch.arange(s["tables"].shape[1], device=DEV)
    live = col < n.unsqueeze(1)
    page = s["tables"][live].long()
    tokens = (s["lens"].long().unsqueeze(1) - col * PAGE)[live]
    valid = torch.arange(PAGE, device=DEV) < tokens.unsqueeze(1)
    rec[page, :, 0], rec[page, :, 1], step[page] = _bounds(s["pool"][page, :, 0], valid.unsqueeze(1))
    return rec, step


def _index(s):
    pages, kv_heads, _, _, dim = s["pool"].shape
    rec, step = _fill_index(s, pages, kv_heads, dim)
    return {"values": (rec.float() * step[:, :, None, None]).to(torch.bfloat16)}


# ---- sparse: score(page) = max over the group's heads of sum_d max(q_d lo_d, q_d hi_d), q in 8 bits too

def _query_steps(q):
    """(whole numbers of magnitude <= 127 as fp32, step) of q [..., d]."""
    q = q.float()
    most = q.abs().amax(-1)
    step = _two_to(torch.frexp(most.clamp_min(2.0 ** -100))[1] - 7)
    return torch.round(q / step.unsqueeze(-1)).clamp(-127, 127), step


def _select(s):
    case = s["case"]
    B, H, K, D, budget = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["budget"]
    rec, step = _index_views(s["index"], s["pool"].shape[0], K, D)
    n = (s["lens"].long() + PAGE - 1) // PAGE
    col = torch.arange(s["tables"].shape[1], device=DEV)
    live = col < n.unsqueeze(1)
    q8, q_step = _query_steps(s["q"].view(B, K, H // K, D))
    page = s["tables"].clamp_min(0).long()
    lo, hi = rec[page].float().transpose(1, 2).unbind(3)      # [B, K, n, D] each
    dots = torch.matmul(q8.clamp_min(0), hi.transpose(-1, -2)) + torch.matmul(q8.clamp_max(0), lo.transpose(-1, -2))
    score = (dots * q_step.unsqueeze(-1) * step[page].transpose(1, 2).unsqueeze(2)).amax(2)
    score = torch.where(live.unsqueeze(1), score, -math.inf)
    kept = live & ((col < case["sink"]) | (col >= (n - case["recent"]).unsqueeze(1)))
    score = torch.where(kept.unsqueeze(1), math.inf, score)
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1][:, :, :budget]
    count = n.clamp_max(budget)
    order = torch.where(torch.arange(order.shape[2], device=DEV) < count[:, None, None], order, col.numel()).sort(-1)[0]
    chosen = torch.gather(s["tables"].unsqueeze(1).expand(B, K, -1), 2, order.clamp_max(col.numel() - 1))
    chosen = torch.where(order < col.numel(), chosen, -1)
    pages = torch.full((B, K, budget), -1, dtype=torch.int32, device=DEV)
    pages[:, :, :chosen.shape[2]] = chosen
    return pages, ((count - 1) * PAGE + s["lens"] - (n - 1) * PAGE).int()


def _sparse(s):
    case = s["case"]
    B, H, K, D = case["batch"], case["heads"], case["kv_heads"], case["dim"]
    pages, lens = _select(s)
    width = max(1, int(pages.ge(0).sum(-1).max()))
    at = pages[:, :, :width].clamp_min(0).long()
    head = torch.arange(K, device=DEV)[None, :, None]
    k = s["pool"][at, head, 0].reshape(B, K, width * PAGE, D).float()
    v = s["pool"][at, head, 1].reshape(B, K, width * PAGE, D).float()
    seen = torch.arange(width * PAGE, device=DEV) < lens[:, None, None, None]
    score = torch.matmul(s["q"].view(B, K, H // K, D).float(), k.transpose(-1, -2)) / math.sqrt(D)
    score = score.masked_fill(~seen, -math.inf)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    out = torch.matmul(w, v) / w.sum(-1, keepdim=True)
    return {"out": out.view(B, H, D).to(torch.bfloat16), "pages": pages, "lens": lens}


# ---- verify: accept while u q(x) < p(x); then a token of max(p - q, 0), or of p after the last draft

def _verify(s):
    target, draft, x = s["target"], s["draft"], s["drafted"].long()
    B, K = x.shape
    row = torch.arange(B, device=DEV)
    n = s["draft_lens"].long() if s["draft_lens"] is not None else torch.full((B,), K, device=DEV)
    p = torch.gather(target[:, :K], 2, x.unsqueeze(-1)).squeeze(-1).double()
    q = torch.gather(draft, 2, x.unsqueeze(-1)).squeeze(-1).double() if draft is not None else torch.ones_like(p)
    ok = (s["u_accept"].double() * q < p) & (torch.arange(K, device=DEV) < n.unsqueeze(1))
    taken = ok.long().cumprod(1).sum(1)
    refused = taken < n
    p_row = target[row, taken].double()
    at = taken.clamp_max(K - 1)
    if draft is not None:
        w = (p_row - draft[row, at].double() * refused.unsqueeze(1)).clamp_min(0)
    else:
        hit = refused.unsqueeze(1) & (torch.arange(p_row.shape[1], device=DEV) == x[row, at].unsqueeze(1))
        w = torch.where(hit, 0.0, p_row)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p_row)
    cdf = w.cumsum(1)
    first = (cdf <= s["u_sample"].double().unsqueeze(1) * cdf[:, -1:]).sum(1)
    last = w.shape[1] - 1 - (w.flip(1) > 0).int().argmax(1)
    token = torch.minimum(first, last)
    col = torch.arange(K + 1, device=DEV)
    drafted = torch.cat((x, x[:, :1]), 1)
    tokens = torch.where(col < taken.unsqueeze(1), drafted, torch.where(col == taken.unsqueeze(1), token.unsqueeze(1), -1))
    return {"tokens": tokens.int(), "accepted": taken.int()}


# ------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "verify":
        B, K, V = case["batch"], case["drafts"], case["vocab"]
        size = 4 if case["dtype"] == "float32" else 2
        # one row of the target's; after a refusal (about half of the requests) one of the draft's too
        rows = 1.5 if case["draft_probs"] else 1.0
        return {"bytes": B * V * size * rows + B * K * (4 + 2 * size) + B * (K + 2) * 4, "flops": 2 * B * V * rows}
    lens, new = _lengths(case)
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    pages = [_pages(n) for n in lens]
    if case["op"] == "rope":
        T = sum(new)
        return {"bytes": T * (H + 2 * K) * D * 2 * 2 + case["rotary"] * 2 + len(lens) * 8 + T * 4, "flops": 3 * T * (H + K) * case["rotary"]}
    if case["op"] == "index":
        n = sum(pages)
        total = n + max(1, n // 50)
        return {"bytes": sum(lens) * K * D * 2 + n * (K * (2 * D + 4) + 4) + total * K * 2 * D * 2, "flops": 2 * sum(lens) * K * D}
    budget = case["budget"]
    scored = sum(n for n in pages if n > budget)
    tokens = sum(min(n, budget) * PAGE - (n * PAGE - length) for n, length in zip(pages, lens))
    small = len(lens) * (2 * H * D * 2 + K * budget * 4 + 8) + sum(pages) * 4
    return {"bytes": scored * K * (2 * D + 4) + tokens * K * 2 * D * 2 + small,
            "flops": scored * H * D * 2 + tokens * H * D * 4}


# ------------------------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    forms = {"rope": _exact_rope, "index": _exact_index, "sparse": _exact_sparse, "verify": _exact_verify}
    return forms[case["op"]](state)


def _exact_rope(s):
    f64, case = torch.float64, s["case"]
    half = case["rotary"] // 2
    pool = s["pool"].to(f64)
    q_out = s["q"].to(f64)
    lens, T = s["lens"].tolist(), s["q"].shape[0]
    starts = s["new_start"].tolist() if s["new_start"] is not None else [r * (T // len(lens)) for r in range(len(lens) + 1)]
    even = torch.arange(half, device=DEV) * 2 if case["interleaved"] else torch.arange(half, device=DEV)
    odd = even + 1 if case["interleaved"] else even + half

    def turned(x, z):
        x = x.to(f64)
        w = torch.complex(x[..., even], x[..., odd]) * z.unsqueeze(1)
        x[..., even], x[..., odd] = w.real, w.imag
        return x

    for r, length in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        if a == b:
            continue
        pos = torch.arange(length - (b - a), length, device=DEV)
        turn = torch.outer(pos.to(f64), s["inv_freq"].to(f64))
        z = torch.polar(torch.ones_like(turn), turn)
        q_out[a:b] = turned(s["q"][a:b], z)
        where = s["tables"][r].long()[pos // PAGE]
        pool[where, :, 0, pos % PAGE] = turned(s["k"][a:b], z)
        pool[where, :, 1, pos % PAGE] = s["v"][a:b].to(f64)
    return {"q": q_out, "pool": pool}


def _power_below(x):
    """The largest power of two that is at most x, for positive normal fp64: x with its fraction bits cleared."""
    return (x.view(torch.int64) >> 52 << 52).view(torch.float64)


def _exact_bounds(keys):
    """(lo, hi, step) in fp64 of keys [n, heads, tokens, d], all of them counted."""
    lo, hi = keys.amin(2), keys.amax(2)
    most = torch.maximum(-lo, hi).amax(-1).clamp_min(2.0 ** -100)
    step = _power_below(most) / 64
    step = torch.where(torch.ceil(most / step) > 127, 2 * step, step)
    return torch.floor(lo / step.unsqueeze(-1)), torch.ceil(hi / step.unsqueeze(-1)), step


def _exact_index(s):
    pages, K, _, _, D = s["pool"].shape
    values = torch.zeros(pages, K, 2, D, dtype=torch.float64, device=DEV)
    for r, length in enumerate(s["lens"].tolist()):
        full, rest = divmod(length, PAGE)
        for ids, tokens in ((s["tables"][r, :full].long(), PAGE), (s["tables"][r, full:full + (rest > 0)].long(), rest)):
            if ids.numel():
                lo, hi, step = _exact_bounds(s["pool"][ids, :, 0, :tokens].double())
                values[ids, :, 0], values[ids, :, 1] = lo * step.unsqueeze(-1), hi * step.unsqueeze(-1)
    return {"values": values}


def _exact_sparse(s):
    case = s["case"]
    B, H, K, D, budget, sink, recent = (case[n] for n in ("batch", "heads", "kv_heads", "dim", "budget", "sink", "recent"))
    G = H // K
    rec, step = _index_views(s["index"], s["pool"].shape[0], K, D)
    out = torch.empty(B, H, D, dtype=torch.float64, device=DEV)
    for r, length in enumerate(s["lens"].tolist()):
        n = _pages(length)
        ids = s["tables"][r, :n].long()
        q = s["q"][r].double().view(K, G, D)
        picks = torch.arange(n, device=DEV).expand(K, n)
        if n > budget:
            most = q.abs().amax(-1).clamp_min(2.0 ** -100)
            q_step = _power_below(most) / 64
            whole = torch.round(q / q_step.unsqueeze(-1)).clamp(-127, 127)
            lo, hi = rec[ids, :, 0].double(), rec[ids, :, 1].double()       # [n, K, D]
            high = torch.einsum("kgd,nkd->kgn", whole.clamp_min(0), hi) + torch.einsum("kgd,nkd->kgn", whole.clamp_max(0), lo)
            score = (high * q_step.unsqueeze(-1) * step[ids].double().t().unsqueeze(1)).amax(1)
            middle = score[:, sink:n - recent]
            best = torch.sort(middle, dim=-1, descending=True, stable=True)[1][:, :budget - sink - recent] + sink
            ends = [i for i in range(n) if i < sink or i >= n - recent]
            picks = torch.cat((best, torch.tensor(ends, device=DEV).expand(K, -1)), 1).sort(-1)[0]
        for h in range(K):
            kv = s["pool"][ids[picks[h]], h].double()                        # [m, 2, 16, D]
            live = (picks[h].unsqueeze(1) * PAGE + torch.arange(PAGE, device=DEV) < length).flatten()
            k, v = kv[:, 0].reshape(-1, D)[live], kv[:, 1].reshape(-1, D)[live]
            out[r, h * G:(h + 1) * G] = torch.softmax(q[h] @ k.t() / math.sqrt(D), -1) @ v
    return {"out": out, "pages": None, "lens": None}


def _exact_verify(s):
    B, K = s["drafted"].shape
    tokens, accepted = torch.full((B, K + 1), -1, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    for b, drafts in enumerate(s["drafted"].tolist()):
        n = K if s["draft_lens"] is None else int(s["draft_lens"][b])
        for j in range(n + 1):
            w = s["target"][b, j].double()
            if j == n:
                break
            x = drafts[j]
            q = torch.zeros_like(w).index_fill(0, torch.tensor(x, device=DEV), 1.0) if s["draft"] is None else s["draft"][b, j].double()
            if float(s["u_accept"][b, j]) * float(q[x]) >= float(w[x]):
                w = w - q if bool((w > q).any()) else w
                w[w < 0] = 0
                break
            tokens[b, j] = x
        up_to = torch.cumsum(w, 0)
        above = torch.nonzero(up_to > float(s["u_sample"][b]) * float(up_to[-1]))
        tokens[b, j] = int(above[0]) if above.numel() else int(torch.nonzero(w > 0)[-1])
        accepted[b] = j
    return {"tokens": tokens.to(DEV), "accepted": accepted.to(DEV)}
