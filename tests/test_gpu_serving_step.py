"""The serving example end to end: prompts, then single tokens, against the same layer in 64 bits.

The reference uses the dequantised weights and unquantised keys and values, so the difference is what 8 bits cost: half a
step of a page's scale (at most max|x| / 254) in every key and value, BF16 between the calls (2^-8 each), and the
softmax of scores that are off by e_s.  A value of the mixture is off by at most its keys' part, 2 e_s max|v|, and
max|v| / 254 + 2^-7 max|v|; the bound below carries that through the output projection with the row sums of |w|.
"""
import importlib.util
import os

import pytest
import torch

from paper_2609_24519_b200 import binding as b

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("serving_step", os.path.join(ROOT, "examples", "serving_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def dense(W):
    codes, scale, _ = W.tensors
    c = codes.to(torch.int16)
    q = torch.stack([((c & 15) ^ 8) - 8, ((c >> 4) ^ 8) - 8], 2).reshape(W.N, W.K).double()
    return q * scale.double().repeat_interleave(W.group, 1)


def test_prompts_then_single_tokens():
    m = load_example()
    layer = m.AttentionLayer(max_tokens=80)
    g = torch.Generator(device="cuda").manual_seed(7)
    w_qkv, w_out = dense(layer.w_qkv), dense(layer.w_out)
    D, Hq, H = layer.dim, layer.q_heads, layer.heads
    past = [[], [], []]
    for new in ([20, 1, 33], [1, 1, 1], [1, 0, 1], [0, 40, 0], [1, 1, 1], [16, 16, 16]):
        x = torch.empty((sum(new), layer.hidden), device="cuda").normal_(generator=g).to(torch.bfloat16)
        y = layer.step(x, new).double()
        qkv = (x.double() @ w_qkv.t()).view(-1, Hq + 2 * H, D)
        at, want, bound = 0, [], []
        for i, n in enumerate(new):
            past[i] += [qkv[at + j] for j in range(n)]
            for j in range(n):
                seen = torch.stack(past[i][:len(past[i]) - n + j + 1])
                out, err = [], []
                for head in range(Hq):
                    kv = head // (Hq // H)
                    q, k, v = qkv[at + j, head], seen[:, Hq + kv], seen[:, Hq + H + kv]
                    s = k @ q * D ** -0.5
                    e_s = float((k.abs().max() / 254 * q.abs().sum() + 2.0 ** -7 * (k.abs() @ q.abs()).max()) * D ** -0.5)
                    out.append(torch.softmax(s, 0) @ v)
                    top = float(v.abs().max())
                    err.append(torch.full((D,), top * (2 * e_s + 1 / 254 + 2.0 ** -7)))
                want.append(w_out @ torch.cat(out))
                bound.append(w_out.abs().cpu() @ torch.cat(err).double())
            at += n
        want, bound = torch.stack(want), torch.stack(bound).cuda() + 2.0 ** -7 * torch.stack(want).abs()
        assert bool(((y - want).abs() <= bound).all())
        # the bound is for the worst case; on the whole the layer is much nearer
        assert float((y - want).norm() / want.norm()) < 0.03
    assert b.awe_last_device_status(layer.h) == (0, 0)
    assert layer.ctx.tolist() == layer.lengths and int((layer.table >= 0).sum()) == layer.n_pages - layer.free.numel()


def test_the_example_runs(capsys):
    load_example().main()
    assert "served [30, 11, 43] tokens" in capsys.readouterr().out
