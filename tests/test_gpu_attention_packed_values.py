"""What is not a number in a packed cache or a query, in every form of the step: it reaches the rows that see it, the weights of the
slots that those rows see, and nothing else."""
import math

import pytest
import torch

from test_gpu_attention import BF, HF, lens_tensor
from test_gpu_attention_packed import lap      # noqa: F401

pytestmark = pytest.mark.gpu

# slots, query heads to a key head, tokens: one workgroup for a cache with its scores in LDS and in the workspace, and chunks, of 16 and 32
# columns and of more rows than a workgroup's
FORMS = [(200, 2, 5), (1000, 2, 5), (4200, 2, 5), (200, 4, 5), (600, 4, 5), (4200, 4, 5), (4200, 16, 4)]
NEAR = dict(rtol=2 ** -6, atol=2 ** -6)


def make(gen, b, h, kv, n, tokens, d, kind):
    k, v = (torch.randn(b, kv, n, d, generator=gen).to(kind) for _ in range(2))
    return k, v, torch.randn(b, h, tokens, d, generator=gen).to(kind).cuda()


@pytest.mark.parametrize("kind,bits,d", [(BF, 4, 128), (HF, 8, 64), (HF, 4, 80)])
@pytest.mark.parametrize("n,group,tokens", FORMS)
def test_values_and_keys(lap, n, group, tokens, kind, bits, d):      # noqa: F811
    b, kv = 2, 2
    gen = torch.Generator().manual_seed(n + group)
    k0, v0, q = make(gen, b, kv * group, kv, n, tokens, d, kind)
    lens, q_lens = [n, n - 77], [tokens, tokens - 2]
    args = dict(lens=lens_tensor(lens), q_lens=lens_tensor(q_lens))
    w = torch.rand(b, kv, n, generator=gen).cuda()
    good = lap.cache_pack(k0.cuda(), v0.cuda(), bits)
    fine = lap.attention_step_packed(q, good["k"], good["v"], w, **args)
    fine = {name: x.cpu().float() for name, x in fine.items()}
    rows = slice(group, 2 * group)      # of key head 1
    in_group = torch.arange(d) // 32 == 1
    for back in (1, 2, tokens - 1, tokens, n // 2):      # slots from the end
        bad = v0.clone()
        for i in range(b):
            bad[i, 1, lens[i] - back, 33] = math.inf
        c = lap.cache_pack(k0.cuda(), bad.cuda(), bits)
        got = {name: x.cpu().float() for name, x in lap.attention_step_packed(q, c["k"], c["v"], w, **args).items()}
        assert torch.equal(got["lse"], fine["lse"]) and torch.equal(got["weights"], fine["weights"]) and torch.equal(got["out"][:, :group], fine["out"][:, :group])
        for i in range(b):
            for t in range(tokens):
                sees = t < q_lens[i] and back >= q_lens[i] - t
                row = got["out"][i, rows, t]
                assert torch.equal(row.isnan(), (in_group & sees).expand(group, d)), (back, i, t)
                assert torch.equal(row[:, ~in_group], fine["out"][i, rows, t][:, ~in_group])
                assert sees or torch.allclose(row, fine["out"][i, rows, t], **NEAR)
        bad = k0.clone()
        for i in range(b):
            bad[i, 1, lens[i] - back, 2] = math.nan
        c = lap.cache_pack(bad.cuda(), v0.cuda(), bits)
        got = {name: x.cpu().float() for name, x in lap.attention_step_packed(q, c["k"], c["v"], w, **args).items()}
        assert torch.equal(got["out"][:, :group], fine["out"][:, :group]) and torch.equal(got["weights"][:, 0], fine["weights"][:, 0])
        for i in range(b):
            for t in range(tokens):
                sees = t < q_lens[i] and back >= q_lens[i] - t
                row, lse = got["out"][i, rows, t], got["lse"][i, rows, t]
                if sees:
                    assert row.isnan().all() and lse.isnan().all(), (back, i, t)
                else:
                    assert torch.allclose(row, fine["out"][i, rows, t], **NEAR) and torch.allclose(lse, fine["lse"][i, rows, t], rtol=1e-5, atol=1e-4)
            # the last token sees all slots in use
            assert got["weights"][i, 1, :lens[i]].isnan().all() and torch.equal(got["weights"][i, 1, lens[i]:], w[i, 1, lens[i]:].cpu())


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("n,group,tokens", FORMS)
def test_weights_of_slots_that_a_row_does_not_see(lap, n, group, tokens, kind):      # noqa: F811
    """A query that is not a number: the slots behind its token receive what the other rows give them."""
    b, kv, d, t = 2, 2, 64, 1
    gen = torch.Generator().manual_seed(n)
    k, v, q = make(gen, b, kv * group, kv, n, tokens, d, kind)
    q[:, ::group, t, 5] = math.nan
    c = lap.cache_pack(k.cuda(), v.cuda(), 8)
    w = torch.rand(b, kv, n, generator=gen).cuda()
    got = lap.attention_step_packed(q, c["k"], c["v"], w)
    held = lap.cache_unpack(c["k"], c["v"], kind, d)
    lse = lap.attention(q, held["k"], held["v"], causal=True)["lse"]
    want = lap.attention_weights(q, held["k"], lse, before=w, causal=True)["weights"]
    seen = n - tokens + t + 1
    assert got["weights"][..., :seen].isnan().all() and want[..., :seen].isnan().all()
    assert torch.isfinite(want[..., seen:]).all() and torch.allclose(got["weights"][..., seen:], want[..., seen:], rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("n,group", [(200, 4), (1000, 8), (4200, 4), (200, 20), (600, 20), (4200, 20), (4200, 70)])
def test_weights_of_empty_slots(lap, n, group, kind):      # noqa: F811
    """A key that is not a number: empty slots, and those past the length, keep the weights that they had."""
    b, kv, d = 2, 2, 64
    gen = torch.Generator().manual_seed(n)
    k, v, q = make(gen, b, kv * group, kv, n, 1, d, kind)
    k[0, 0, 7] = k[1, 1, n // 2] = math.nan
    c = lap.cache_pack(k.cuda(), v.cuda(), 4)
    pos = torch.arange(n, dtype=torch.int32).expand(b, kv, n).clone()
    pos[torch.rand(b, kv, n, generator=gen) < 0.3] = -1
    pos[0, 0, 7] = pos[1, 1, n // 2] = 3
    lens = [n, n - 5]
    w = torch.rand(b, kv, n, generator=gen).cuda()
    got = lap.attention_step_packed(q[:, :, 0], c["k"], c["v"], w, lens=lens_tensor(lens), positions=pos.cuda())["weights"]
    for i in range(b):
        for j in range(kv):
            used = ((pos[i, j] >= 0) & (torch.arange(n) < lens[i])).cuda()
            assert torch.equal(got[i, j, ~used], w[i, j, ~used])
            assert got[i, j, used].isnan().all() if i == j else torch.isfinite(got[i, j]).all()
