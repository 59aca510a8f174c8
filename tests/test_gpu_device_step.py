"""The operators together, as a serving loop uses them: pages are handed out, tokens rotated and appended to the 8-bit
cache, attention reads it through a window, logits become probabilities, drafts are verified, and what was rejected
gives its pages back -- captured once in a graph and replayed, with nothing on the host between the steps."""
import numpy as np
import pytest
import torch

import ref_step as ref
from paper_2501_08090_b200 import binding as b

pytestmark = pytest.mark.gpu

HQ, HKV, D, V, DRAFTS, WINDOW, SINK = 8, 2, 64, 413, 3, 40, 4


class Model:
    """One attention layer between an embedding and a vocabulary projection (random weights); drafts come from a bigram table."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.embed = torch.randn(V, (HQ + 2 * HKV) * D, generator=g, device="cuda").to(torch.bfloat16)
        self.head = (0.4 * torch.randn(HQ * D, V, generator=g, device="cuda")).to(torch.bfloat16)
        self.next = torch.randint(0, V, (V,), generator=g, device="cuda", dtype=torch.int32)
        self.freq = (10000.0 ** (-torch.arange(D // 2, device="cuda") / (D // 2))).float()

    def qkv(self, tokens):
        x = self.embed[tokens.long()].view(-1, HQ + 2 * HKV, D)
        return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]


def test_a_speculative_step_in_a_graph():
    torch.manual_seed(0)
    model, prompts, steps = Model(1), [70, 5, 33, 1, 0], 12
    B, N = len(prompts), DRAFTS + 1
    prompts[4] = 16
    width = ref.pages(max(prompts) + (steps + 2) * N)
    pages = sum(ref.pages(n + (steps + 2) * N) for n in prompts) + 2
    kp = b.Kv8Pool(b.make_config(1, HQ, HKV, D, pages, width, B))
    kp.pool.fill_(0x5a)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    tables, lens, count = i32(B, width) - 1, i32(B), torch.full((1,), pages, dtype=torch.int32, device="cuda")
    free = torch.randperm(pages, device="cuda", dtype=torch.int32)
    text = torch.randint(0, V, (B, max(prompts) + (steps + 2) * N), device="cuda", dtype=torch.int32)
    texts = [text[r, :n + 1].tolist() for r, n in enumerate(prompts)]         # n cached tokens and the one that is fed next

    # the prompts, in one call each
    new = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    start, step_lens, slots = i32(B + 1), i32(B), torch.zeros(sum(prompts), dtype=torch.int64, device="cuda")
    kp.pages_assign(tables, lens, new, free, count, lens_out=lens, count_out=count, step_lens=step_lens, new_start=start, slots=slots)
    q, k, v = model.qkv(torch.tensor([t for x in texts for t in x[:-1]], device="cuda"))
    kp.kv8_append(0, tables, step_lens, k, v, q=q, q_out=torch.empty_like(q), inv_freq=model.freq, new_start=start)
    assert len(set(slots.tolist())) == sum(prompts)

    # one step, on buffers that stay where they are
    last = torch.tensor([x[-1] for x in texts], dtype=torch.int32, device="cuda")
    grow, params = i32(B) + N, torch.tensor([1.1, 0.2, 0.1, 0.8], device="cuda").repeat(B, 1)
    history_lens, prompt_lens = torch.tensor([len(x) for x in texts], dtype=torch.int32, device="cuda"), torch.tensor([len(x) for x in texts], dtype=torch.int32, device="cuda")
    mask = torch.full((B, N, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    mask[0, :, 3] = 0                                        # request 0 may not say tokens 96 .. 127
    turned = torch.empty(B * N, HQ, D, dtype=torch.bfloat16, device="cuda")
    attended = torch.empty(B, N, HQ, D, dtype=torch.bfloat16, device="cuda")
    probs = torch.empty(B, N, V, device="cuda")
    tokens, accepted, drafts = i32(B, N), i32(B), i32(B, DRAFTS)
    ua, us, logits = torch.zeros(B, DRAFTS, device="cuda"), torch.zeros(B, device="cuda"), torch.empty(B, N, V, device="cuda")
    keep, col = i32(B), torch.arange(N, device="cuda")

    def step():
        t = last
        for i in range(DRAFTS):
            t = model.next[t.long()]
            drafts[:, i] = t
        kp.pages_assign(tables, lens, grow, free, count, lens_out=lens, count_out=count, step_lens=step_lens)
        q, k, v = model.qkv(torch.cat((last[:, None], drafts), 1).flatten())
        kp.kv8_append(0, tables, step_lens, k, v, q=q, q_out=turned, inv_freq=model.freq)
        kp.kv8_attention(0, tables, step_lens, turned.view(B, N, HQ, D), attended, window=WINDOW, sink=SINK)
        logits.copy_((attended.flatten(2) @ model.head).float())
        b.logits_process(logits, probs, params=params, history=text, prompt_lens=prompt_lens, history_lens=history_lens, drafts=drafts, mask=mask)
        b.draft_verify(drafts, probs, None, ua, us, tokens, accepted)
        torch.sub(lens, DRAFTS - accepted, out=keep)          # what was rejected leaves the cache
        kp.pages_release(tables, lens, keep, free, count, lens_out=lens, count_out=count)
        at = torch.where(col <= accepted[:, None], history_lens[:, None] + col, text.shape[1] - 1)
        text.scatter_(1, at.long(), torch.where(col <= accepted[:, None], tokens, text[:, -1:]))
        history_lens.add_(accepted + 1)
        last.copy_(torch.gather(tokens, 1, accepted[:, None].long())[:, 0])

    # the cache beside it in numpy
    def quantised(seq_of_calls):
        rec, steps_ = np.zeros((width, HKV, 2, 16, D)), np.zeros((width, HKV, 2))
        for length, rows in seq_of_calls:
            ref.append8_tokens(rec, steps_, list(range(width)), length, rows)
        return rec, steps_

    from paper_2501_08090_b200.binding import KvPool
    plain = KvPool(b.make_config(1, HQ, HKV, D, B * width, width, B))         # keys as kv_append_rope turns them
    own_tables = torch.arange(B * width, device="cuda", dtype=torch.int32).view(B, width)

    def turned_rows(r, first, toks):
        q, k, v = model.qkv(torch.tensor(toks, device="cuda"))
        sl = i32(B)
        sl[:] = 1
        sl[r] = first + len(toks)
        start = i32(B + 1)
        start[r + 1:] = len(toks)
        plain.kv_append_rope(0, own_tables, sl, None, k, v, None, model.freq, new_start=start)
        t = np.arange(first, first + len(toks))
        pool = plain.pool_view()[0].double().cpu().numpy()
        return pool[own_tables[r].cpu().numpy()[t // 16], :, :, t % 16]

    calls = [[(n, turned_rows(r, 0, texts[r][:-1]))] if n else [] for r, n in enumerate(prompts)]
    graph, g = torch.cuda.CUDAGraph(), torch.Generator(device="cuda").manual_seed(3)
    total = 0
    for i in range(steps):
        before = lens.tolist()
        ua.copy_(torch.rand(B, DRAFTS, generator=g, device="cuda") ** 3 * (0.02 if i % 2 else 1.0))            # every other step lenient
        us.copy_(torch.rand(B, generator=g, device="cuda"))
        if i == 1:
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                step()
        graph.replay() if i else step()
        torch.cuda.synchronize()
        assert kp.check_status() == 0
        got, acc, drafted = tokens.tolist(), accepted.tolist(), drafts.tolist()
        for r in range(B):
            fed = [texts[r][-1]] + drafted[r]
            calls[r].append((before[r] + N, turned_rows(r, before[r], fed)))
            rec, st = quantised(calls[r])
            L = before[r] + N
            t = np.arange(L)
            kv = rec[t // 16, :, :, t % 16] * st[t // 16][..., None]
            qs = turned.view(B, N, HQ, D)[r].double().cpu().numpy()
            out = attended[r].double().cpu().numpy()
            for h in range(HKV):
                want, size, mass, floor = ref.attend(qs[:, h * 4:h * 4 + 4], kv[:, h, 0], kv[:, h, 1], L, WINDOW, SINK, st[t // 16, h, 1])
                assert np.all(np.abs(out[:, h * 4:h * 4 + 4] - want) <= ref.attend_tolerance(want, size, mass, 11, floor)), (i, r, h)
            x = logits[r].double().cpu().numpy()
            allowed = np.ones(V, bool)
            allowed[96:128] = r != 0
            for j in range(N):
                _, p = ref.logits(x[j], params[r].tolist(), texts[r][:prompts[r] + 1], texts[r][prompts[r] + 1:] + drafted[r][:j], (), allowed)
                assert np.abs(probs[r, j].double().cpu().numpy() - p).max() <= 2e-6
            n = acc[r]
            assert got[r][:n] == drafted[r][:n] and got[r][n + 1:] == [-1] * (DRAFTS - n) and (r or not 96 <= got[r][n] < 128)
            texts[r] += got[r][:n + 1]
            total += n
        assert lens.tolist() == [x + 1 + n for x, n in zip(before, acc)] and history_lens.tolist() == [len(x) for x in texts]
        assert [text[r, :len(x)].tolist() for r, x in enumerate(texts)] == texts
        held = [p for r, n in enumerate(lens.tolist()) for p in tables[r, :ref.pages(n)].tolist()] + free[:int(count)].tolist()
        assert sorted(held) == list(range(pages))
    assert total > 0
    plain.close()
    kp.close()


def test_arguments_that_do_not_fit_are_named():
    """Every tensor of every call: of another type, shape, layout or device, or none at all, it is refused by its name."""
    B, T, H, K, P = 3, 6, 8, 2, 5
    cfg = b.make_config(1, H, K, D, 20, P, 4)
    pool, pool8 = b.KvPool(cfg), b.Kv8Pool(cfg)

    def ints(*shape, dtype=torch.int32):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    def rows(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")

    step = dict(block_tables=ints(B, P), seq_lens=ints(B))
    pages = dict(step, free_pages=ints(20), free_count=ints(1), lens_out=ints(B), count_out=ints(1))
    calls = [
        (pool.pages_assign, dict(pages, new_tokens=ints(B), step_lens=ints(B), new_start=ints(B + 1), slots=ints(7, dtype=torch.int64)), {}),
        (pool8.pages_release, dict(pages, keep_lens=ints(B)), {}),
        (pool.decode_attention_window, dict(step, q=rows(B, 2, H, D), out=rows(B, 2, H, D)), dict(layer=0, window=5)),
        (pool8.kv8_attention, dict(step, q=rows(B, H, D), out=rows(B, H, D)), dict(layer=0)),
        (pool8.kv8_append, dict(step, k_new=rows(T, K, D), v_new=rows(T, K, D), q=rows(T, H, D), q_out=rows(T, H, D),
                                inv_freq=torch.zeros(16, device="cuda"), new_start=ints(B + 1)), dict(layer=0)),
        (pool8.kv8_gather, dict(step, k=rows(T, K, D), v=rows(T, K, D), start=ints(B + 1)), dict(layer=0))]
    sparse = torch.zeros(B, device="cuda").to_sparse()
    for call, tensors, others in calls:
        call(**tensors, **others)
        for name, t in tensors.items():
            wrong = [t.cpu(), t.to(torch.float16), t[None, None], 5, "x", sparse]
            if name not in ("slots", "inv_freq", "seq_lens", "q", "k_new", "k"):         # others follow the sizes of these
                wrong.append(torch.cat([t, t]))
            if name != "seq_lens" and t.numel() > 1:
                wrong.append(torch.stack([t, t], -1)[..., 0])                            # elements apart
            for w in wrong:
                with pytest.raises(ValueError) as e:
                    call(**dict(tensors, **{name: w}), **others)
                assert "must be" in str(e.value) or "go together" in str(e.value)
                if "must be" in str(e.value) and name not in ("seq_lens", "q", "k_new", "k"):
                    assert str(e.value).startswith(name + " must be"), (call.__name__, name, e.value)
        if "layer" in others:
            with pytest.raises(OverflowError):
                call(**tensors, **dict(others, layer=1 << 40))
    with pytest.raises(ValueError):
        pool8.kv8_append(0, **dict(calls[4][1], q_out=None))
    pool.close()
    with pytest.raises(b.CkvError):
        pool.decode_attention_window(0, window=5, **calls[2][1])
    torch.cuda.synchronize()
