"""Attention over a packed cache where scaled scores are so large that numbers of 32 bits stand far apart: what a row's largest score
comes to must not depend on how its product with the scale is rounded."""
import math

import pytest
import torch

import attention_ref as ref
from test_gpu_attention import BF, HF, lens_tensor, within
from test_gpu_attention_packed import lap      # noqa: F401

pytestmark = pytest.mark.gpu

# slots, rows of queries to a key head: one workgroup for a cache with its scores in LDS and in the workspace, and chunks, of 16 and 32 columns
FORMS = [(100, 4), (1000, 8), (4200, 4), (100, 20), (500, 20), (4200, 20), (300, 70)]
# scale (None: 1 / sqrt(d)), about what q.k comes to
SIZES = [(1e6, 100.7), (None, 2.4e9), (1e6, 3000.0), (1.0, 0.7)]


def equal_keys(gen, b, kv, n, d, kind, about):
    """Keys that are all one row, values as they come, and queries (of b sequences, one head) whose products with that row are near `about`."""
    side = math.sqrt(about / d)
    key = ((0.5 + torch.rand(d, generator=gen)) * side).to(kind)
    v = torch.randn(b, kv, n, d, generator=gen).to(kind)
    return key, v, lambda heads: ((0.5 + torch.rand(b, heads, d, generator=gen)) * side).to(kind).cuda()


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("scale,about", SIZES)
@pytest.mark.parametrize("n,group", FORMS)
def test_equal_scores(lap, n, group, scale, about, kind):      # noqa: F811
    """Every slot has the same key: probabilities are one over the slots in use, and the only slot's is one."""
    b, kv, d = 3, 2, 128
    gen = torch.Generator().manual_seed(n + group)
    key, v, queries = equal_keys(gen, b, kv, n, d, kind, about)
    c = lap.cache_pack(key.expand(b, kv, n, d).contiguous().cuda(), v.cuda(), 8)
    held = lap.cache_unpack(c["k"], c["v"], kind, d)
    kn, vn = held["k"].cpu().double(), held["v"].cpu().double()
    lens, q, w = [1, n, n - 33], queries(kv * group), torch.rand(b, kv, n, generator=gen).cuda()
    got = lap.attention_step_packed(q, c["k"], c["v"], w, lens=lens_tensor(lens), scale=scale)
    for i, m in enumerate(lens):
        mean, size = (x[i, :, :m].mean(1).repeat_interleave(group, 0) for x in (vn, vn.abs()))
        if m == 1:      # a probability of one: nothing is rounded
            assert torch.equal(got["out"][i].cpu().double(), mean)
            assert torch.equal(got["weights"][i, :, :1], w[i, :, :1] + group)
        within(got["out"][i], mean, ref.U[kind] * mean.abs() + ref.E * size + 2.0 ** -25, "out")
        # the product, and its own with the scale, are off by a few 2^-24 of themselves
        x = (scale or d ** -0.5) * (q[i].cpu().double().view(kv, group, d) @ kn[i, :, 0, :, None]).view(-1)
        within(got["lse"][i], x + math.log(m), ref.E * (1 + x), "lse")
        was = w[i].cpu().double()
        added = torch.where(torch.arange(n) < m, group / m, 0.0).expand(kv, n)
        within(got["weights"][i], was + added, ref.E * added + 1e-6 * (1 + was), "weights")


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("scale,about", SIZES[:3])
@pytest.mark.parametrize("n,group", FORMS)
def test_one_slot_takes_all(lap, n, group, scale, about, kind):      # noqa: F811
    """A key half as large again as all others, whose scores are then beyond reach: its value comes out, and its weight is one."""
    b, kv, d = 2, 2, 128
    gen = torch.Generator().manual_seed(n + group)
    key, v, queries = equal_keys(gen, b, kv, n, d, kind, about)
    k = key.expand(b, kv, n, d).clone()
    slot = 2 * n // 3
    k[:, :, slot] *= 1.5
    c = lap.cache_pack(k.cuda(), v.cuda(), 8)
    held = lap.cache_unpack(c["k"], c["v"], kind, d)
    q, w = queries(kv * group), torch.rand(b, kv, n, generator=gen).cuda()
    got = lap.attention_step_packed(q, c["k"], c["v"], w, scale=scale)
    assert torch.equal(got["out"], held["v"][:, :, slot].repeat_interleave(group, 1))
    want = w.clone()
    want[:, :, slot] += group
    assert torch.equal(got["weights"], want)
    assert torch.isfinite(got["lse"]).all()
