"""Measured cases of the operators of a decode step whose state stays on the GPU, around a cache in 8 bits.

Four operators, each in a plain torch form (`own` false) and as the call a user makes of the
library (`own` true):

  append   Kv8Pool.kv8_append: new queries and keys rotated by their positions, keys and values written to an
           8-bit cache in steps of a power of two per page, head and side; then Kv8Pool.kv8_gather of what it wrote.
  attend   Kv8Pool.kv8_attention over that cache, and KvPool.decode_attention_window over the bf16 cache: one or a
           few new tokens per request, the whole context or a sliding window and the first tokens.
  pages    KvPool.pages_release and pages_assign: finished requests' pages return to the free list, new tokens get
           theirs; block tables, lengths, token lists and slot maps.
  logits   logits_process: penalties for repeated tokens, biases and grammar masks on logits, and the
           probabilities that draft_verify reads.

Shapes are this repository's workloads' (8B and 70B head layouts, the small one of its tests) or generic.
`prepare` makes the inputs on the GPU from the seed alone.
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
        dict(name="append_one_token", op="append", batch=1, heads=32, kv_heads=8, dim=128, rotary=128, interleaved=False,
             new_lo=1, new_hi=1, ctx_lo=4100, ctx_hi=4100, packed=True),
        # speculative decoding: five new tokens for each request of the 70B-shaped batch
        dict(name="append_drafts_b96", op="append", batch=96, heads=64, kv_heads=8, dim=128, rotary=128, interleaved=False,
             new_lo=5, new_hi=5, ctx_lo=1024, ctx_hi=4096, packed=True),
        # ragged prompts entering the cache, some as continuation chunks, half of each head rotated in pairs
        dict(name="append_prompts_b8", op="append", batch=8, heads=32, kv_heads=8, dim=128, rotary=64, interleaved=True,
             new_lo=37, new_hi=8191, ctx_lo=0, ctx_hi=12001, packed=False),
        # the small head layout, three tokens a request, short contexts, a window and sinks over the 8-bit cache
        dict(name="attend8_small_b5", op="attend", cache="int8", batch=5, q_len=3, heads=4, kv_heads=1, dim=64,
             ctx_lo=3, ctx_hi=2999, window=512, sink=4),
        # one request with a long context: latency and bandwidth of one stream
        dict(name="attend8_one_131072", op="attend", cache="int8", batch=1, q_len=1, heads=32, kv_heads=8, dim=128,
             ctx_lo=131072, ctx_hi=131072, window=0, sink=0),
        # a full batch on the 8B shape, contexts that differ sixteenfold
        dict(name="attend8_b64", op="attend", cache="int8", batch=64, q_len=1, heads=32, kv_heads=8, dim=128,
             ctx_lo=1024, ctx_hi=16384, window=0, sink=0),
        # a window over one long context of the 70B shape in bf16: latency
        dict(name="window_one_100001", op="attend", cache="bf16", batch=1, q_len=1, heads=64, kv_heads=8, dim=128,
             ctx_lo=100001, ctx_hi=100001, window=1024, sink=4),
        # a batch of a model with sliding windows, bf16, all contexts longer than the window
        dict(name="window_b64", op="attend", cache="bf16", batch=64, q_len=1, heads=32, kv_heads=8, dim=128,
             ctx_lo=4096, ctx_hi=16384, window=2048, sink=4),
        # a decode step of a full interactive instance: one token each, a few requests have finished
        dict(name="pages_decode_b256", op="pages", batch=256, ctx_lo=1, ctx_hi=8191, new_lo=1, new_hi=1, done=8),
        # ragged prompts are admitted while others have finished: pages and slots of every token
        dict(name="pages_prompts_b64", op="pages", batch=64, ctx_lo=0, ctx_hi=4096, new_lo=37, new_hi=2047, done=16),
        # one request's four drafts against a full-size vocabulary: latency
        dict(name="logits_one", op="logits", batch=1, rows=5, vocab=128256, dtype="bfloat16", out="float32", history=4096,
             bias=0, mask=False, penalties=True),
        # an interactive batch with drafts, odd vocabulary, grammar masks, biases and penalties
        dict(name="logits_b128", op="logits", batch=128, rows=4, vocab=50257, dtype="float32", out="float32", history=1500,
             bias=17, mask=True, penalties=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "pages", "logits"])
    if op == "pages":
        batch, most = _log_int(rng, 1, 1024), _log_int(rng, 1, 2047)
        most = max(1, min(most, 64000 // batch))
        ctx = max(1, min(_log_int(rng, 1, 16384), 2000000 // batch))
        return dict(op=op, batch=batch, ctx_lo=rng.randint(0, ctx), ctx_hi=ctx, new_lo=rng.randint(0, most), new_hi=most,
                    done=rng.randint(0, batch // 2))
    if op == "logits":
        batch, rows, vocab = _log_int(rng, 1, 256), rng.randint(1, 8), _log_int(rng, 1000, 151936)
        batch = max(1, min(batch, int(2.5e7 / (rows * vocab))))
        return dict(op=op, batch=batch, rows=rows, vocab=vocab, dtype=rng.choice(["float32", "bfloat16"]),
                    out=rng.choice(["float32", "float32", "bfloat16"]), history=_log_int(rng, 1, 8192),
                    bias=rng.choice([0, 1, 30, 300]), mask=rng.random() < 0.5, penalties=rng.random() < 0.7)
    heads, kv_heads, dim = rng.choice([(32, 8, 128), (64, 8, 128), (8, 2, 128), (4, 1, 64), (12, 4, 64), (6, 6, 128), (35, 5, 128)])
    case = dict(op=op, batch=_log_int(rng, 1, 96), heads=heads, kv_heads=kv_heads, dim=dim)
    if op == "append":
        ragged = rng.random() < 0.5
        most = _log_int(rng, 1, 8191) if ragged else rng.randint(1, 8)
        case["batch"] = max(1, min(case["batch"], int(1400000 * 128 / (most * (heads + 2 * kv_heads) * dim))))
        low = rng.randint(0, most) if ragged else most
        ctx = max(1, min(_log_int(rng, 1, 20000), 400000 // case["batch"]))
        case.update(rotary=rng.choice([0, dim, dim // 2, 16]), interleaved=rng.random() < 0.5, new_lo=low, new_hi=most,
                    ctx_lo=rng.randint(0, ctx), ctx_hi=ctx, packed=rng.random() < 0.5)
        return case
    q_len = rng.choice([1, 1, 1, 2, 5])
    ctx = _log_int(rng, q_len, 131072)
    case["batch"] = max(1, min(case["batch"], int(500000 * 1024 / (ctx * kv_heads * dim))))
    window = rng.choice([0, _log_int(rng, 1, 4096)])
    cache = rng.choice(["int8", "int8", "bf16"])
    if cache == "bf16" and window == 0:
        window = _log_int(rng, 16, 4096)
    case.update(cache=cache, q_len=q_len, ctx_lo=rng.randint(q_len, ctx), ctx_hi=ctx, window=window,
                sink=rng.choice([0, 1, 4, 100]) if window else 0)
    return case


# ------------------------------------------------------------------------------------ the inputs

def _spread(lo, hi, n):
    """n whole numbers from lo to hi, the same for every seed (what is read depends on their sum)."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _pages(length):
    return (length + PAGE - 1) // PAGE


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(counts):
    return torch.tensor([0] + counts, device=DEV).cumsum(0).to(torch.int32)


def _rows(shape, gen):
    """Keys as a model's are: pages with a direction of their own, a few large channels; values plain."""
    x = torch.randn(shape, generator=gen, device=DEV)
    x[:, :, 0] += 0.7 * torch.randn(shape[0], shape[1], 1, shape[-1], generator=gen, device=DEV)
    x[:, :, 0, :, ::31] *= 3.0
    return x


def _tables(counts, gen):
    """(block tables, pages of the pool): every request's pages anywhere in the pool."""
    total = sum(counts)
    pages = total + max(1, total // 50)
    order = torch.randperm(pages, generator=gen, device=DEV, dtype=torch.int32)
    tables = torch.full((len(counts), max(1, max(counts))), -1, dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(counts):
        tables[r, :n] = order[at:at + n]
        at += n
    return tables, pages


def _cache8(pages, kv_heads, dim, gen):
    """(the 8-bit cache's bytes, its records, its steps): filled a part at a time."""
    records_n = pages * kv_heads * 2 * PAGE * dim
    cache = torch.zeros(records_n + pages * kv_heads * 8, dtype=torch.uint8, device=DEV)
    records, steps = _views8(cache, pages, kv_heads, dim)
    for at in range(0, pages, 4096):
        n = min(4096, pages - at)
        rows = _rows((n, kv_heads, 2, PAGE, dim), gen).to(torch.bfloat16).float()
        step = _step(rows.abs().amax((-1, -2)))
        steps[at:at + n] = step
        records[at:at + n] = torch.round(rows / step[..., None, None]).clamp(-127, 127).to(torch.int8)
    return cache, records, steps


def _views8(cache, pages, kv_heads, dim):
    cut = pages * kv_heads * 2 * PAGE * dim
    return cache[:cut].view(torch.int8).view(pages, kv_heads, 2, PAGE, dim), cache[cut:].view(torch.float32).view(pages, kv_heads, 2)


def _config(case, state, pages):
    from paper_2501_08090_b200 import binding
    return binding.make_config(1, case.get("heads", 8), case.get("kv_heads", 2), case.get("dim", 64), pages, state["tables"].shape[1],
                               case["batch"])


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"case": case}
    return {"append": _prepare_append, "attend": _prepare_attend, "pages": _prepare_pages, "logits": _prepare_logits}[case["op"]](case, state, gen)


def _shuffled(lists, gen):
    mix = torch.randperm(len(lists[0]), generator=gen, device=DEV).tolist()
    return [[x[i] for i in mix] for x in lists]


def _append_lengths(case):
    """(lengths after the step, new tokens, tokens gathered afterwards) of the requests."""
    ctx = _spread(case["ctx_lo"], case["ctx_hi"], case["batch"])
    new = _spread(case["new_lo"], case["new_hi"], case["batch"])[::-1]
    lens = [c + n for c, n in zip(ctx, new)]
    return lens, new, [min(c, PAGE - 1) + n for c, n in zip(ctx, new)]


def _prepare_append(case, state, gen):
    lens, new, back = _shuffled(_append_lengths(case), gen)
    H, K, D, T = case["heads"], case["kv_heads"], case["dim"], sum(new)
    state["tables"], pages = _tables([_pages(n) for n in lens], gen)
    state["lens"] = _ints(lens)
    state["cache"], state["records"], state["steps"] = _cache8(pages, K, D, gen)
    if case["packed"]:         # one projection gives queries, keys and values side by side
        qkv = torch.randn(T, H + 2 * K, D, generator=gen, device=DEV).to(torch.bfloat16)
        state["q"], state["k"], state["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
    else:
        state["q"], state["k"], state["v"] = (torch.randn(T, h, D, generator=gen, device=DEV).to(torch.bfloat16) for h in (H, K, K))
    state["inv_freq"], half = None, case["rotary"] // 2
    if half:
        state["inv_freq"] = (500000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)).float()
    state["new_start"] = _starts(new) if min(new) != max(new) else None
    state["back_start"] = _starts(back)
    state["touched"] = sum(_pages(n) - (n - m) // PAGE for n, m in zip(lens, new) if m)
    state["q_out"] = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
    state["k_out"], state["v_out"] = (torch.empty(sum(back), K, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if own:
        from paper_2501_08090_b200 import binding
        state["handle"] = binding.Kv8Pool(_config(case, state, pages), device="cuda:0", pool=state["cache"])
    return state


def _prepare_attend(case, state, gen):
    B, H, K, D, N = case["batch"], case["heads"], case["kv_heads"], case["dim"], case["q_len"]
    lens, = _shuffled([_spread(case["ctx_lo"], case["ctx_hi"], B)], gen)
    state["tables"], pages = _tables([_pages(n) for n in lens], gen)
    state["lens"] = _ints(lens)
    if case["cache"] == "int8":
        state["cache"], state["records"], state["steps"] = _cache8(pages, K, D, gen)
    else:
        state["pool"] = torch.empty(pages, K, 2, PAGE, D, dtype=torch.bfloat16, device=DEV)
        for at in range(0, pages, 4096):
            state["pool"][at:at + 4096] = _rows((min(4096, pages - at), K, 2, PAGE, D), gen)
    q = torch.randn(B, N, H, D, generator=gen, device=DEV)
    q += 0.7 * torch.randn(B, N, 1, D, generator=gen, device=DEV)
    state["q"] = q.to(torch.bfloat16)
    state["out"] = torch.empty(B, N, H, D, dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2501_08090_b200 import binding
        cfg = _config(case, state, pages)
        if case["cache"] == "int8":
            state["handle"] = binding.Kv8Pool(cfg, device="cuda:0", pool=state["cache"])
        else:
            state["handle"] = binding.KvPool(cfg, device="cuda:0", pool=state["pool"].view(-1))
    return state


def _page_lengths(case):
    """(lengths before, lengths kept, new tokens) of the requests; the first `done` are finished or cut back."""
    B, done = case["batch"], case["done"]
    lens = _spread(case["ctx_lo"], case["ctx_hi"], B)[::-1]
    new = _spread(case["new_lo"], case["new_hi"], B)
    keep = [(0 if r % 3 else n // 2) if r < done else n for r, n in enumerate(lens)]
    return lens, keep, [0 if r < done else n for r, n in enumerate(new)]


def _prepare_pages(case, state, gen):
    lens, keep, new = _shuffled(_page_lengths(case), gen)
    B, T = case["batch"], sum(new)
    held = [_pages(n) for n in lens]
    width = max(1, max(_pages(n + m) for n, m in zip(lens, new)))
    spare = sum(_pages(n + m) - h for n, m, h in zip(lens, new, held)) + 5
    order = torch.randperm(sum(held) + spare, generator=gen, device=DEV, dtype=torch.int32)
    tables = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    live = torch.arange(width, device=DEV) < _ints(held).unsqueeze(1)
    tables[live] = order[:sum(held)]
    free = torch.full((order.numel(),), -1, dtype=torch.int32, device=DEV)
    free[:spare] = order[sum(held):]
    state.update(tables=tables, lens=_ints(lens), keep=_ints(keep), new=_ints(new), free=free, free_count=_ints([spare]))
    for name in ("kept_lens", "lens_out", "step_lens"):
        state[name] = torch.empty(B, dtype=torch.int32, device=DEV)
    state["kept_count"], state["count_out"] = (torch.empty(1, dtype=torch.int32, device=DEV) for _ in range(2))
    state["new_start"] = torch.empty(B + 1, dtype=torch.int32, device=DEV)
    state["slots"] = torch.empty(T, dtype=torch.int64, device=DEV)
    if own:
        from paper_2501_08090_b200 import binding
        state["handle"] = binding.KvPool(_config(case, state, order.numel()), device="cuda:0")
    return state


def _prepare_logits(case, state, gen):
    B, R, V, most = case["batch"], case["rows"], case["vocab"], case["history"]
    state["logits"] = torch.empty(B, R, V, dtype=getattr(torch, case["dtype"]), device=DEV)
    for b in range(0, B, 32):
        state["logits"][b:b + 32] = 2.5 * torch.randn(min(32, B - b), R, V, generator=gen, device=DEV)
    state["out"] = torch.empty(B, R, V, dtype=getattr(torch, case["out"]), device=DEV)

    def text(*shape):          # a few tokens come again and again, as in text
        return (torch.rand(*shape, generator=gen, device=DEV) ** 4 * V).int().clamp_max(V - 1)

    state["options"] = {}
    if case["penalties"]:
        unit = torch.rand(B, 4, generator=gen, device=DEV)
        params = unit * torch.tensor([0.4, 1.0, 0.5, 0.9], device=DEV) + torch.tensor([1.0, -0.2, 0.0, 0.4], device=DEV)
        params[1::7, 3] = 0.0  # some requests take the best token
        lens = torch.tensor(_spread((most + 1) // 2, most, B), dtype=torch.int32, device=DEV)[torch.randperm(B, generator=gen, device=DEV)]
        prompts = (lens * torch.rand(B, generator=gen, device=DEV)).int()
        state["options"].update(params=params, history=text(B, most), prompt_lens=prompts, history_lens=lens)
        if R > 1:
            state["options"]["drafts"] = text(B, R - 1)
    if case["bias"]:
        ids = text(B, case["bias"])
        ids[:, 1::5] = -1      # requests have fewer biases than there is room for
        state["options"].update(bias_ids=ids, bias=4 * torch.randn(B, case["bias"], generator=gen, device=DEV))
    if case["mask"]:
        words = torch.randint(-2 ** 31, 2 ** 31, (B, R, (V + 31) // 32), generator=gen, device=DEV, dtype=torch.int64).int()
        words[::3] &= torch.randint(-2 ** 31, 2 ** 31, words[::3].shape, generator=gen, device=DEV, dtype=torch.int64).int()
        words[1::3] = -1       # no grammar here
        words[2::11, R - 1] = 0                                           # a dead end: nothing is allowed
        state["options"]["mask"] = words
    return state


# ------------------------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _run_own(op, state)
    return {"append": _append, "attend": _attend, "pages": _release_assign, "logits": _logits}[op](state)


def _run_own(op, s):
    case = s["case"]
    if op == "logits":
        from paper_2501_08090_b200 import binding
        binding.logits_process(s["logits"], s["out"], **s["options"])
        return {"out": s["out"]}
    kp = s["handle"]
    if op == "append":
        turned = s["inv_freq"] is not None
        kp.kv8_append(0, s["tables"], s["lens"], s["k"], s["v"], q=s["q"] if turned else None, q_out=s["q_out"] if turned else None,
                      inv_freq=s["inv_freq"], new_start=s["new_start"], interleaved=case["interleaved"])
        kp.kv8_gather(0, s["tables"], s["lens"], s["k_out"], s["v_out"], start=s["back_start"])
        return {"q": s["q_out"] if turned else s["q"], "k": s["k_out"], "v": s["v_out"]}
    if op == "attend":
        if case["cache"] == "int8":
            kp.kv8_attention(0, s["tables"], s["lens"], s["q"], s["out"], window=case["window"], sink=case["sink"])
        else:
            kp.decode_attention_window(0, s["tables"], s["lens"], s["q"], s["out"], window=case["window"], sink=case["sink"])
        return {"out": s["out"]}
    kp.pages_release(s["tables"], s["lens"], s["keep"], s["free"], s["free_count"], lens_out=s["kept_lens"], count_out=s["kept_count"])
    kp.pages_assign(s["tables"], s["kept_lens"], s["new"], s["free"], s["kept_count"], lens_out=s["lens_out"], count_out=s["count_out"],
                    step_lens=s["step_lens"], new_start=s["new_start"], slots=s["slots"])
    return _page_outputs(s)


def _page_outputs(s):
    return {n: s[n] for n in ("tables", "free", "kept_lens", "kept_count", "lens_out", "count_out", "step_lens", "new_start", "slots")}


# ---- append: x' = x cos(a) - y sin(a), y' = y cos(a) + x sin(a), a = position * inv_freq; then whole steps of a power of two

def _two_to(exp):
    """2^exp as fp32, for whole exponents of normal numbers (a power function may be off by a rounding)."""
    return ((exp.int() + 127) << 23).view(torch.float32)


def _step(most):
    """The step of a block whose largest magnitude is `most`: between most / 128 and most / 64."""
    return _two_to(torch.frexp(most.clamp_min(2.0 ** -100))[1] - 7)


def _rotate(x, cos, sin, half, interleaved):
    x = x.float()
    a, b, rest = (x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]) if interleaved else \
        (x[..., :half], x[..., half:2 * half], x[..., 2 * half:])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((ra, rb), -1).flatten(-2) if interleaved else torch.cat((ra, rb), -1)
    return torch.cat((turned, rest), -1).to(torch.bfloat16)


def _tokens(starts, lens, T):
    """(request, position) of each row of a list of every request's last tokens."""
    i = torch.arange(T, device=DEV)
    r = torch.searchsorted(starts, i, right=True) - 1
    return r, lens[r] - (starts[r + 1] - i)


def _append(s):
    T, lens, q, k = s["q"].shape[0], s["lens"].long(), s["q"], s["k"]
    B, K, D = lens.numel(), k.shape[1], k.shape[2]
    starts = torch.arange(B + 1, device=DEV) * (T // B) if s["new_start"] is None else s["new_start"].long()
    r, pos = _tokens(starts, lens, T)
    if s["inv_freq"] is not None:
        angle = pos.double().unsqueeze(-1) * s["inv_freq"].double()
        cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
        half, inter = s["inv_freq"].numel(), s["case"]["interleaved"]
        q, k = _rotate(q, cos, sin, half, inter), _rotate(k, cos, sin, half, inter)
    column, slot = pos // PAGE, pos % PAGE
    first = torch.ones(T, dtype=torch.bool, device=DEV)
    first[1:] = (r[1:] != r[:-1]) | (column[1:] != column[:-1])
    block, P = first.cumsum(0) - 1, s["touched"]
    page = torch.zeros(P, dtype=torch.int64, device=DEV)
    page[block] = s["tables"][r, column].long()
    fresh = torch.zeros(P, PAGE, dtype=torch.bool, device=DEV)
    fresh[block, slot] = True
    rows = torch.zeros(P, PAGE, K, 2, D, device=DEV)
    rows[block, slot] = torch.stack((k.float(), s["v"].float()), 2)
    rows = rows.permute(0, 2, 3, 1, 4)                                    # [P, K, 2, 16, D], as the cache
    step, before = _step(rows.abs().amax((-1, -2))), s["steps"][page]
    step = torch.where(fresh[:, 0].view(P, 1, 1), step, torch.maximum(step, before))
    old = s["records"][page]
    moved = torch.round(old.float() * (before / step)[..., None, None])
    kept = torch.where((torch.arange(PAGE, device=DEV) < fresh.int().argmax(1, keepdim=True)).view(P, 1, 1, PAGE, 1), moved, old.float())
    here = torch.round(rows / step[..., None, None]).clamp(-127, 127)
    s["records"][page] = torch.where(fresh.view(P, 1, 1, PAGE, 1), here, kept).to(torch.int8)
    s["steps"][page] = step
    back = s["back_start"].long()
    r, pos = _tokens(back, lens, s["k_out"].shape[0])
    page, slot = s["tables"][r, pos // PAGE].long(), pos % PAGE
    values = (s["records"][page, :, :, slot].float() * s["steps"][page].unsqueeze(-1)).to(torch.bfloat16)
    return {"q": q, "k": values[:, :, 0], "v": values[:, :, 1]}


# ---- attend: out = softmax(q k / sqrt(d)) v over t <= pos with t > pos - window or t < sink

def _attend(s):
    case = s["case"]
    B, N, H, D = s["q"].shape
    K, lens = case["kv_heads"], s["lens"].long()
    width, window, sink = s["tables"].shape[1], case["window"] or 1 << 30, case["sink"]
    tail = min(width, (window + N + PAGE - 2) // PAGE + 1)                # pages that hold the windows, from the last one back
    head = min(width, _pages(sink))
    last = (lens - 1) // PAGE
    column = torch.cat((torch.arange(head, device=DEV).expand(B, head), last.unsqueeze(1) - torch.arange(tail - 1, -1, -1, device=DEV)), 1)
    in_tail = torch.arange(head + tail, device=DEV) >= head
    page = torch.gather(s["tables"], 1, column.clamp(0, width - 1)).clamp_min(0).long()
    if case["cache"] == "int8":
        k, v = (s["records"][page][:, :, :, i].float() * s["steps"][page][:, :, :, i, None, None] for i in (0, 1))
    else:
        k, v = (s["pool"][page][:, :, :, i].float() for i in (0, 1))      # [B, n, K, 16, D]
    k, v = (x.transpose(1, 2).reshape(B, K, -1, D) for x in (k, v))
    t = (column.unsqueeze(-1) * PAGE + torch.arange(PAGE, device=DEV)).view(B, 1, -1)
    pos = (lens.unsqueeze(1) - N + torch.arange(N, device=DEV)).unsqueeze(-1)
    near = (t > pos - window) & (t <= pos) & (t >= 0) & in_tail.repeat_interleave(PAGE)
    seen = near | ((t < sink) & (t <= pos - window) & ~in_tail.repeat_interleave(PAGE))          # [B, N, tokens]
    q = s["q"].float().view(B, N, K, H // K, D).permute(0, 2, 3, 1, 4).reshape(B, K, -1, D)      # columns: head of the group, new token
    score = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D)
    score = score.masked_fill(~seen.unsqueeze(1).repeat(1, 1, H // K, 1), -math.inf)
    w = torch.exp(score - score.amax(-1, keepdim=True))
    out = torch.matmul(w, v) / w.sum(-1, keepdim=True)
    return {"out": out.view(B, K, H // K, N, D).permute(0, 3, 1, 2, 4).reshape(B, N, H, D).to(torch.bfloat16)}


# ---- pages: a stack of free pages; what a list of requests gives back or takes lies in order of request and context

def _flat(counts, total):
    """(request, index within it) of `total` entries, counts[r] for each request r in turn."""
    ends = counts.cumsum(0)
    i = torch.arange(total, device=DEV)
    r = torch.searchsorted(ends, i, right=True)
    return r, i - (ends - counts)[r]


def _release_assign(s):
    lens, keep, new, tables, free = s["lens"].long(), s["keep"].long(), s["new"].long(), s["tables"], s["free"]
    held, kept = (lens + PAGE - 1) // PAGE, (keep + PAGE - 1) // PAGE
    B, width = tables.shape
    gone = held - kept
    column = torch.arange(width, device=DEV)
    leaves = (column >= kept.unsqueeze(1)) & (column < held.unsqueeze(1))
    order = (gone.cumsum(0) - gone - kept).unsqueeze(1) + column          # the k-th page to go
    count = s["free_count"].long()
    room = torch.zeros(free.numel() + 1, dtype=torch.int32, device=DEV)
    room[torch.where(leaves, count + gone.sum() - 1 - order, free.numel())] = tables
    place = torch.arange(free.numel(), device=DEV)
    free.copy_(torch.where((place >= count) & (place < count + gone.sum()), room[:-1], free))
    count = count + gone.sum()
    s["kept_lens"].copy_(keep)
    s["kept_count"].copy_(count)
    need = (keep + new + PAGE - 1) // PAGE - kept
    upto = need.cumsum(0)
    served = (need == 0) | (upto <= count)
    takes = served.unsqueeze(1) & (column >= kept.unsqueeze(1)) & (column < (kept + need).unsqueeze(1))
    order = (upto - need - kept).unsqueeze(1) + column
    tables.copy_(torch.where(takes, free[(count - 1 - order).clamp(0, free.numel() - 1)], tables))
    after = torch.where(served, keep + new, keep)
    s["lens_out"].copy_(after)
    s["count_out"].copy_(count - (need * served).sum())
    s["step_lens"].copy_(torch.where(served, after, 0))
    s["new_start"][0] = 0
    s["new_start"][1:] = new.cumsum(0)
    r, i = _flat(new, s["slots"].numel())
    pos = keep[r] + i
    slot = tables[r, (pos // PAGE).clamp_max(width - 1)].long() * PAGE + pos % PAGE
    s["slots"].copy_(torch.where(served[r], slot, -1))
    return _page_outputs(s)


# ---- logits: penalties by how often a token came, biases, masks; exp((x - max) / T) / sum

def _counts(ids, valid, V):
    """How often each token stands among the valid ones of ids [B, n]: [B, V]."""
    at = torch.where(valid & (ids >= 0) & (ids < V), ids, V).long()
    return torch.zeros(ids.shape[0], V + 1, device=DEV).scatter_add_(1, at, torch.ones_like(at, dtype=torch.float32))[:, :V]


def _logits(s):
    o, (B, R, V) = s["options"], s["logits"].shape
    x = s["logits"].float()
    temperature = torch.ones(B, 1, 1, device=DEV)
    if "params" in o:
        place = torch.arange(o["history"].shape[1], device=DEV)
        told, prompt = place < o["history_lens"].unsqueeze(1), place < o["prompt_lens"].unsqueeze(1)
        made = _counts(o["history"], told & ~prompt, V).unsqueeze(1).repeat(1, R, 1)
        if R > 1:
            drafted = torch.zeros(B, R, V + 1, device=DEV)
            drafted[:, 1:].scatter_(2, o["drafts"].long().unsqueeze(-1), 1.0)
            made += drafted[..., :V].cumsum(1)
        seen = (made > 0) | (_counts(o["history"], told & prompt, V) > 0).unsqueeze(1)
        rep, pres, freq, temperature = (o["params"][:, i].view(B, 1, 1) for i in range(4))
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x = x - freq * made - pres * (made > 0)
    if "bias" in o:            # where an id stands twice, the last entry counts
        at = torch.where((o["bias_ids"] >= 0) & (o["bias_ids"] < V), o["bias_ids"], V).long()
        entry = torch.arange(1, at.shape[1] + 1, device=DEV).expand_as(at)
        entry = torch.zeros(B, V + 1, dtype=torch.int64, device=DEV).scatter_reduce_(1, at, entry, "amax")[:, :V]
        added = torch.gather(o["bias"], 1, (entry - 1).clamp_min(0))
        x = x + torch.where(entry > 0, added, 0.0).unsqueeze(1)
    if "mask" in o:
        bit = (o["mask"].unsqueeze(-1) >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        x = x.masked_fill(bit.flatten(-2)[..., :V] == 0, -math.inf)
    most = x.amax(-1, keepdim=True)
    dead = most == -math.inf
    w = torch.exp((x - most.masked_fill(dead, 0.0)) / torch.where(temperature > 0, temperature, 1.0))
    best = torch.zeros_like(w).scatter_(2, (x == most).int().argmax(-1, keepdim=True), 1.0)
    p = torch.where(temperature > 0, w / w.sum(-1, keepdim=True), best)
    return {"out": torch.where(dead, 0.0, p).to(s["out"].dtype)}


# ------------------------------------------------------------------------------------ what a pass cannot do without

def _visible(length, N, window, sink):
    """Tokens that some of a request's N new tokens see."""
    first = max(0, length - N - window + 1) if window else 0
    return length - first + min(first, sink)


def work(case):
    op, B = case["op"], case["batch"]
    if op == "logits":
        R, V = case["rows"], case["vocab"]
        size = {"float32": 4, "bfloat16": 2}
        bytes_ = B * R * V * (size[case["dtype"]] + size[case["out"]])
        if case["penalties"]:
            bytes_ += 4 * sum(_spread((case["history"] + 1) // 2, case["history"], B)) + B * (24 + 4 * (R - 1))
        return {"bytes": bytes_ + B * case["bias"] * 8 + (B * R * ((V + 31) // 32) * 4 if case["mask"] else 0), "flops": 6 * B * R * V}
    if op == "pages":
        lens, keep, new = _page_lengths(case)
        moved = sum(_pages(n) - _pages(k) + _pages(k + m) - _pages(k) for n, k, m in zip(lens, keep, new))
        return {"bytes": moved * 8 + sum(new) * 8 + B * 4 * 7 + 16, "flops": 0}
    H, K, D = case["heads"], case["kv_heads"], case["dim"]
    if op == "append":
        lens, new, back = _append_lengths(case)
        T, S = sum(new), sum(back)
        pages = sum(_pages(n) - (n - m) // PAGE for n, m in zip(lens, new) if m)
        moved = T * (H * 2 * (2 if case["rotary"] else 0) + 2 * K * 3) * D + pages * (K * 8 + 4)
        return {"bytes": moved + S * 2 * K * D * 3 + pages * K * 8 + B * 8, "flops": 3 * T * (H + K) * case["rotary"] + 4 * T * K * D}
    N = case["q_len"]
    tokens = sum(_visible(n, N, case["window"], case["sink"]) for n in _spread(case["ctx_lo"], case["ctx_hi"], B))
    row = 2 * D + 8 / PAGE if case["cache"] == "int8" else 4 * D
    return {"bytes": tokens * K * row + tokens / PAGE * 4 + B * (N * H * D * 4 + 4), "flops": 4 * tokens * N * H * D}


# ------------------------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    state = prepare(case, seed)
    forms = {"append": _exact_append, "attend": _exact_attend, "pages": lambda s: None, "logits": _exact_logits}
    return forms[case["op"]](state)


def _power_below(x):
    """The largest power of two that is at most x, for positive normal fp64: x with its fraction bits cleared."""
    return (x.view(torch.int64) >> 52 << 52).view(torch.float64)


def _exact_append(s):
    f64, case = torch.float64, s["case"]
    half, lens, T = case["rotary"] // 2, s["lens"].tolist(), s["q"].shape[0]
    starts = s["new_start"].tolist() if s["new_start"] is not None else [r * (T // len(lens)) for r in range(len(lens) + 1)]
    back = s["back_start"].tolist()
    q_out = s["q"].to(f64)
    out = torch.empty(2, back[-1], case["kv_heads"], case["dim"], dtype=f64, device=DEV)
    even = torch.arange(half, device=DEV) * 2 if case["interleaved"] else torch.arange(half, device=DEV)
    odd = even + 1 if case["interleaved"] else even + half

    def turned(x, z):
        x = x.to(f64)
        w = torch.complex(x[..., even], x[..., odd]) * z.unsqueeze(1)
        x[..., even], x[..., odd] = w.real, w.imag
        return x

    for r, length in enumerate(lens):
        a, b = starts[r], starts[r + 1]
        if back[r] == back[r + 1]:
            continue
        p0, first = length - (b - a), length - (back[r + 1] - back[r])
        k, v = s["k"][a:b].to(f64), s["v"][a:b].to(f64)
        if half and b > a:
            turn = torch.outer(torch.arange(p0, length, device=DEV).to(f64), s["inv_freq"].to(f64))
            z = torch.polar(torch.ones_like(turn), turn)
            q_out[a:b] = turned(s["q"][a:b], z)
            k = turned(k, z).to(torch.bfloat16).to(f64)                   # the cache is given what a bf16 cache would hold
        base = p0 // PAGE * PAGE                                          # the first page that changes
        n = _pages(length) - base // PAGE
        ids = s["tables"][r].long()[base // PAGE:base // PAGE + n]
        rows = torch.zeros(n * PAGE, 2, *k.shape[1:], dtype=f64, device=DEV)
        rows[p0 - base:length - base] = torch.stack((k, v), 1)
        rows = rows.view(n, PAGE, 2, *k.shape[1:])
        step = _power_below(rows.abs().amax((1, 4)).clamp_min(2.0 ** -100)) / 64              # [n, 2, K]
        value = torch.round(rows / step[:, None, :, :, None]).clamp(-127, 127) * step[:, None, :, :, None]
        if p0 > base:                                                     # the page that older tokens share
            was = s["steps"][ids[0]].to(f64).t()
            both = torch.maximum(step[0], was)
            value[0] = torch.round(rows[0] / both[None, :, :, None]).clamp(-127, 127) * both[None, :, :, None]
            old = s["records"][ids[0]].to(f64)[:, :, :p0 - base].permute(2, 1, 0, 3)
            value[0, :p0 - base] = torch.round(old * (was / both)[None, :, :, None]) * both[None, :, :, None]
        value = value.view(n * PAGE, 2, *k.shape[1:])
        at = torch.arange(first, length, device=DEV)
        page, slot = s["tables"][r].long()[at // PAGE], at % PAGE
        whole = s["records"][page, :, :, slot].to(f64) * s["steps"][page].to(f64).unsqueeze(-1)                # [tokens, K, 2, D]
        whole[at >= base] = value[at[at >= base] - base].transpose(1, 2)
        out[:, back[r]:back[r + 1]] = whole.permute(2, 0, 1, 3)
    return {"q": q_out, "k": out[0], "v": out[1]}


def _exact_attend(s):
    case, q = s["case"], s["q"].double()
    B, N, H, D = q.shape
    K, window, sink = case["kv_heads"], case["window"], case["sink"]
    out = torch.empty(B, N, H, D, dtype=torch.float64, device=DEV)
    for r, length in enumerate(s["lens"].tolist()):
        ids = s["tables"][r, :_pages(length)].long()
        for i in range(N):
            p = length - N + i
            t = torch.arange(max(0, p - window + 1) if window else 0, p + 1, device=DEV)
            t = torch.cat((torch.arange(min(sink, int(t[0])), device=DEV), t))
            page, slot = ids[t // PAGE], t % PAGE
            for h in range(K):
                if case["cache"] == "int8":
                    kv = s["records"][page, h, :, slot].double() * s["steps"][page, h].double().unsqueeze(-1)
                else:
                    kv = s["pool"][page, h, :, slot].double()
                G = H // K
                w = torch.softmax(q[r, i, h * G:(h + 1) * G] @ kv[:, 0].t() / math.sqrt(D), -1)
                out[r, i, h * G:(h + 1) * G] = w @ kv[:, 1]
    return {"out": out}


def _exact_logits(s):
    o, (B, R, V) = s["options"], s["logits"].shape
    out = torch.zeros(B, R, V, dtype=torch.float64, device=DEV)
    for b in range(B):
        rep, pres, freq, temp = o["params"][b].tolist() if "params" in o else (1.0, 0.0, 0.0, 1.0)
        said, heard = [], torch.empty(0, dtype=torch.int64, device=DEV)
        if "params" in o:
            n, m = int(o["prompt_lens"][b]), int(o["history_lens"][b])
            heard, said = o["history"][b, :n].long(), [o["history"][b, n:m].long()]
        for j in range(R):
            x = s["logits"][b, j].double()
            if "params" in o:
                if j:
                    said.append(o["drafts"][b, j - 1:j].long())
                count = torch.bincount(torch.cat(said), minlength=V).double()
                known = torch.unique(torch.cat((heard, *said)))
                x[known] = torch.where(x[known] > 0, x[known] / rep, x[known] * rep)
                x -= freq * count + pres * count.clamp_max(1.0)
            if "bias" in o:
                last = {}
                for token, value in zip(o["bias_ids"][b].tolist(), o["bias"][b].tolist()):
                    last[token] = value
                last.pop(-1, None)
                x[list(last)] += torch.tensor(list(last.values()), dtype=torch.float64, device=DEV)
            allowed = torch.ones(V, dtype=torch.bool, device=DEV)
            if "mask" in o:
                v = torch.arange(V, device=DEV)
                allowed = (o["mask"][b, j].long()[v // 32] >> (v % 32)) % 2 != 0
            if not bool(allowed.any()):
                continue
            x = torch.where(allowed, x, -math.inf)
            out[b, j] = torch.softmax(x / temp, 0) if temp > 0 else (torch.arange(V, device=DEV) == x.argmax()).double()
    return {"out": out}
