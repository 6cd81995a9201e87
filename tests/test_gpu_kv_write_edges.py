"""The 8-bit cache write over lists with skipped slots: the stored bytes and scales are specified, so they are equal."""
import numpy as np
import pytest
import torch

from paper_2609_24519_b200 import binding as b
from tests.gpu_util import handle
from tests.test_gpu_kv_cache import TYPES, cuda

pytestmark = pytest.mark.gpu


def plain_write(cache, scale, x, slots, page):
    """Page by page, in FP32 with the specified roundings; finite rows."""
    f = np.float32
    fine = (slots >= 0) & (slots < cache.shape[0] * page)
    for p in np.unique(slots[fine] // page):
        t = np.flatnonzero(fine & (slots // page == p))
        place = int(slots[t[0]] % page)
        rows = x[t].astype(f)  # tokens, heads, dimensions
        a = np.abs(rows).max((0, 2))
        wanted = np.where(a < f(2.0 ** -100), f(0), a * (f(1) / f(127)))
        before = scale[p] if place else np.zeros_like(wanted)
        after = np.maximum(before, wanted)
        for h in np.flatnonzero(after > before):
            if place:
                cache[p, h, :place] = np.rint(cache[p, h, :place].astype(f) * (before[h] / after[h])).astype(np.int8)
        inverse = np.where(after > 0, f(1) / np.where(after > 0, after, f(1)), f(0))
        q = np.clip(np.rint(rows * inverse[:, None]), -127, 127).astype(np.int8)
        for i, s in enumerate(slots[t]):
            cache[p, :, s % page] = q[i]
        scale[p] = after


def run(rng, slots, n_pages, heads, dim, page, kind, ld_extra):
    T, ld = len(slots), 2 * heads * dim + ld_extra
    x = torch.from_numpy(rng.standard_normal((T, ld)).astype(np.float32) * np.exp(rng.standard_normal((T, 1)))).to(TYPES[kind][1])
    x[slots < 0] = float("nan")  # what is skipped is not looked at
    caches = [rng.integers(-127, 128, (n_pages, heads, page, dim)).astype(np.int8) for _ in range(2)]
    scales = [np.abs(rng.standard_normal((n_pages, heads))).astype(np.float32) * 0.01 for _ in range(2)]
    dev = [cuda(c) for c in caches + scales]
    dx = x.cuda()
    b.awe_kv_write(handle(), b.kv_cache(*dev, n_pages, heads, page, dim), dx, dx[:, heads * dim:], TYPES[kind][0], T, ld, ld, cuda(slots))
    for i in range(2):
        plain_write(caches[i], scales[i], x[:, i * heads * dim:(i + 1) * heads * dim].float().numpy().reshape(T, heads, dim), slots, page)
    for want, got in zip(caches + scales, dev):
        assert np.array_equal(want, got.cpu().numpy())


def filled(rng, cached, new, page):
    """Slots of requests that hold `cached` tokens and add `new`, over shuffled pages."""
    need = [-(-(c + n) // page) for c, n in zip(cached, new)]
    pages, at, slots = rng.permutation(sum(need) + 3), 0, []
    for c, n, k in zip(cached, new, need):
        slots += [int(pages[at + pos // page]) * page + pos % page for pos in range(c, c + n)]
        at += k
    return np.array(slots, np.int64), sum(need) + 3


@pytest.mark.parametrize("heads,dim,page,kind", [(2, 64, 16, "bf16"), (8, 128, 16, "f16"), (4, 128, 64, "bf16"), (1, 256, 256, "f16"), (3, 64, 128, "bf16")])
@pytest.mark.parametrize("share", [0.05, 0.5, 0.9])  # of the tokens that are masked
@pytest.mark.parametrize("ld_extra", [0, 3])
def test_masked_tokens_between_those_of_a_page(heads, dim, page, kind, share, ld_extra):
    rng = np.random.default_rng(heads * dim + page)
    slots, n_pages = filled(rng, [0, 5, page - 1, 3 * page + 7, 2], [2 * page + 3, 3 * page, page + 2, 700, 1], page)
    slots[rng.random(len(slots)) < share] = -1
    slots[[0, 7]] = n_pages * page, -2 ** 62  # outside the pool, at either end
    run(rng, slots, n_pages, heads, dim, page, kind, ld_extra)


@pytest.mark.parametrize("page", [16, 64, 256])
def test_a_page_of_skipped_tokens_between_two_of_a_page(page):
    """As many as may stand there, in lists that windows of every size are taken from."""
    rng = np.random.default_rng(page)
    slots = np.concatenate([np.full(3, -1), [2 * page + 3], np.full(page, -1), [2 * page + 5, 2 * page + 6], np.full(page, -7), [2 * page + 9], [0, 1],
                            np.full(page - 1, -1), [2], np.full(2 * page, -1)])
    run(rng, slots.astype(np.int64), 4, 2, 64, page, "f16", 0)


def test_masked_tokens_in_a_long_list():
    rng = np.random.default_rng(3)
    slots, n_pages = filled(rng, [7, 0, 100], [9000, 3000, 5000], 32)
    slots[rng.random(len(slots)) < 0.2] = -1
    run(rng, slots, n_pages, 2, 64, 32, "bf16", 0)


def test_a_list_of_nothing_but_skipped_slots():
    rng = np.random.default_rng(4)
    run(rng, np.full(500, -1, np.int64), 2, 1, 64, 16, "f16", 0)
