"""The adapter example end to end: each operator's result against 64 bits from what went into it, step by step.

Tolerances.  A 4-bit linear layer or the adapters: FP32 sums (K 2^-23 of the sum of magnitudes) and one rounding to BF16, 2^-8 (the adapters add
to what is rounded already).  Queries: one rounding, 2^-8, and 2^-22 of FP32.  Stored keys and values: half a scale, which is at most
(hi - lo) / 15 (1 + 2^-6).  Attention from what is stored: weights 2^-10, output 2^-8.  Log probabilities as in their own test."""
import importlib.util
import os

import pytest
import torch

from paper_2609_24519_b200 import binding as b

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("adapter_decode", os.path.join(ROOT, "examples", "adapter_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(W):
    codes, scale, _ = W.tensors
    c = codes.to(torch.int16)
    q = torch.stack([((c & 15) ^ 8) - 8, ((c >> 4) ^ 8) - 8], 2).reshape(W.N, W.K).double()
    return q * scale.double().repeat_interleave(W.group, 1)


def near(got, want, slack):
    return bool(((got.double() - want).abs() <= slack).all())


def test_every_operator_of_prompts_and_single_tokens():
    m = load_example()
    model = m.AdapterModel(max_tokens=80)
    g = torch.Generator(device="cuda").manual_seed(7)
    w_qkv, w_out, w_head = dense(model.w_qkv), dense(model.w_out), dense(model.w_head)
    A, B, scale = model.adapters.tensors
    D, Hq, H, page = model.dim, model.q_heads, model.heads, model.page
    table = model.turn.tensors[0].double()
    for new, which in (([20, 1, 33], [0, -1, 1]), ([1, 1, 1], [1, 1, -1]), ([1, 0, 1], [0, 0, 0]), ([0, 40, 0], [1, 1, 1]), ([16, 16, 16], [-1, 0, 1])):
        x = torch.empty((sum(new), model.hidden), device="cuda").normal_(generator=g).to(torch.bfloat16)
        before = list(model.lengths)
        ids, logprob = model.step(x, new, torch.tensor(which, dtype=torch.int32, device="cuda"))
        T = sum(new)
        request = [i for i, n in enumerate(new) for _ in range(n)]
        pos = torch.tensor([before[i] + j for i, n in enumerate(new) for j in range(n)], device="cuda")
        assert torch.equal(model.positions[:T].long(), pos) and model.ctx.tolist() == model.lengths
        # projection and adapters
        xd = x.double()
        qkv = xd @ w_qkv.t()
        slack = 2.0 ** -8 * qkv.abs() + 512 * 2.0 ** -23 * (xd.abs() @ w_qkv.abs().t())
        for t, i in enumerate(request):
            if which[i] >= 0:
                j, f = which[i], float(scale[which[i]])
                u = f * (A[j].double() @ xd[t])
                part = B[j].double() @ u
                u_off = f * 512 * 2.0 ** -23 * (A[j].double().abs() @ xd[t].abs()) + 2.0 ** -15 * u.abs().max()
                slack[t] += 2.0 ** -8 * (qkv[t] + part).abs() + B[j].double().abs() @ u_off + 2.0 ** -8 * slack[t]
                qkv[t] += part
        keys_values = model.qkv[:T].double()[:, (Hq + H) * D:]  # values are not touched any more
        assert near(keys_values, qkv[:, (Hq + H) * D:], 1.01 * slack[:, (Hq + H) * D:])
        # rotation: of the exact rows, so that it inherits their slack
        heads, off = qkv.view(T, Hq + 2 * H, D), slack.view(T, Hq + 2 * H, D)
        cos, sin = table[pos][:, None, :D // 2], table[pos][:, None, D // 2:]
        a, c = heads[:, :Hq + H, :D // 2], heads[:, :Hq + H, D // 2:]
        turned = torch.cat([a * cos - c * sin, c * cos + a * sin], 2)
        a, c = off[:, :Hq + H, :D // 2], off[:, :Hq + H, D // 2:]
        turned_off = torch.cat([a * cos.abs() + c * sin.abs(), c * cos.abs() + a * sin.abs()], 2) * 1.01 + 2.0 ** -20 * turned.abs().amax(2, keepdim=True)
        q = model.qkv[:T].view(T, Hq + 2 * H, D)[:, :Hq]
        assert near(q, turned[:, :Hq], turned_off[:, :Hq] + 2.0 ** -8 * (turned[:, :Hq].abs() + turned_off[:, :Hq]))
        # what is stored
        k, v = (torch.empty((T, H, D), dtype=torch.float16, device="cuda") for _ in range(2))
        b.awe_kv4_read(model.h, model.cache, T, model.slots, b.F16, k, H * D, v, H * D)
        for got, want, far in ((k, turned[:, Hq:], turned_off[:, Hq:]), (v, model.qkv[:T].double().view(T, -1, D)[:, Hq + H:], torch.zeros(T, H, D, device="cuda"))):
            step = (want.amax(2).clamp(min=0) - want.amin(2).clamp(max=0) + 2 * far.amax(2)) / 15 * (1 + 2.0 ** -6)
            assert near(got, want, far + step[..., None] * (0.5 + 2.0 ** -10))
        # attention over the stored values
        qd, at = q.double(), 0
        for i, n in enumerate(new):
            length = model.lengths[i]
            slots = (model.table[i, torch.arange(length, device="cuda") // page].long() * page + torch.arange(length, device="cuda") % page)
            ks, vs = (torch.empty((length, H, D), dtype=torch.float16, device="cuda") for _ in range(2))
            if length:
                b.awe_kv4_read(model.h, model.cache, length, slots, b.F16, ks, H * D, vs, H * D)
            for j in range(n):
                seen = before[i] + j + 1
                for head in range(Hq):
                    kd, vd = ks[:seen, head // (Hq // H)].double(), vs[:seen, head // (Hq // H)].double()
                    p = torch.softmax(kd @ qd[at + j, head] * D ** -0.5, 0)
                    want = p @ vd
                    got = model.mixed[at + j, head * D:(head + 1) * D]
                    assert near(got, want, 2.0 ** -8 * want.abs() + (2.0 ** -10 + 2.0 ** -16) * 1.01 * (p @ vd.abs()))
            at += n
        # the head, and what it says
        rows = model.mixed[:T].double() @ w_out.t()
        assert near(model.rows[:T], rows, 2.0 ** -8 * rows.abs() + 512 * 2.0 ** -23 * (model.mixed[:T].double().abs() @ w_out.abs().t()))
        logits = model.rows[:T].double() @ w_head.t()
        assert near(model.logits[:T], logits, 512 * 2.0 ** -23 * (model.rows[:T].double().abs() @ w_head.abs().t()))
        logp = torch.log_softmax(model.logits[:T].double(), 1)
        order = torch.sort(model.logits[:T], dim=1, descending=True, stable=True).indices[:, :model.alternatives]
        assert torch.equal(ids.long(), order) and near(logprob, logp.gather(1, order), 1e-4)
        assert near(model.entropy[:T], -(logp.exp() * logp).sum(1), 1e-4)
    assert b.awe_last_device_status(model.h) == (0, 0)
    assert int((model.table >= 0).sum()) == model.n_pages - model.free.numel()


def test_the_example_runs(capsys):
    load_example().main()
    assert "answered 11 tokens each after [20, 1, 33]" in capsys.readouterr().out


def test_a_decode_step_in_a_graph():
    """The whole step captured once and replayed with other rows and lengths gives what a call gives."""
    m = load_example()
    one, two = m.AdapterModel(), m.AdapterModel()
    g = torch.Generator(device="cuda").manual_seed(3)
    draw = lambda n: torch.empty((n, one.hidden), device="cuda").normal_(generator=g).to(torch.bfloat16)  # noqa: E731
    adapter = torch.tensor([1, -1, 0], dtype=torch.int32, device="cuda")
    prompt = draw(30)
    for model in (one, two):
        model.step(prompt, [10, 15, 5], adapter)
    x = draw(3)
    new = torch.ones(3, dtype=torch.int32, device="cuda")
    T, h, D = 3, two.h, two.dim

    def calls():
        b.awe_kv_plan(h, two.cached, new, two.B, two.page, two.free, two.free.numel(), two.table, two.max_pages, two.max_pages, two.slots, two.positions, T,
                      two.start, two.ctx, two.counts)
        b.awe_linear_w4(h, two.w_qkv, x, b.BF16, T, x.stride(0), two.qkv, b.BF16, two.width)
        b.awe_linear_adapters(h, two.adapters, x, T, x.stride(0), two.start, adapter, two.B, two.qkv, two.width, two.qkv, b.BF16, two.width)
        b.awe_kv4_append(h, two.cache, two.turn, b.BF16, T, two.q_heads, two.qkv, two.width, two.qkv[:, two.q_heads * D:], two.width,
                         two.qkv[:, (two.q_heads + two.heads) * D:], two.width, two.positions, two.slots, two.qkv, two.width)
        b.awe_kv4_attention(h, two.cache, two.qkv, b.BF16, T, two.q_heads, two.width, two.start, two.ctx, two.B, two.table, two.max_pages, two.max_pages,
                            D ** -0.5, True, 0, two.mixed, two.q_heads * D, None, two.workspace)
        b.awe_linear_w4(h, two.w_out, two.mixed, b.BF16, T, two.q_heads * D, two.rows, b.BF16, two.hidden)
        b.awe_linear_w4(h, two.w_head, two.rows, b.BF16, T, two.hidden, two.logits, b.F32, two.vocabulary)
        b.awe_token_logprobs(h, two.logits, b.F32, T, two.vocabulary, two.vocabulary, 1.0, None, None, two.entropy, None, two.alternatives, two.top_logprob,
                             two.top_id)

    calls()  # warmed up: the same step again writes the same again
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        calls()
    for _ in range(3):
        x.copy_(draw(3))
        ids, logprob = one.step(x, [1, 1, 1], adapter)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, two.top_id[:3]) and torch.equal(logprob, two.top_logprob[:3])
        taken = int(two.counts[0])
        assert taken == 0 or taken <= 3
        two.cached.copy_(two.ctx)
        if taken:  # the graph reads the free list's place, so its entries move instead
            two.free[:-taken].copy_(two.free[taken:].clone())
