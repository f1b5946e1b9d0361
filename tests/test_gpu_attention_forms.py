"""Every form of the kernels that the sharing rules choose, at both widths (up to 64 elements, up to 128), both types, causal,
with a window and without a mask, against 64 bits.  The rules are repeated here, so that a case that no longer reaches the form
that it is for is seen."""
import pytest
import torch

import attention_ref as ref
import test_gpu_attention as ordinary
from test_gpu_attention import BF, HF, lens_tensor, rows, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lap():
    import paper_1903_06631_amd as lap
    lap.load_library()
    return lap


def share(batch, heads, length, causal):
    """Waves of a workgroup, blocks of 32 rows by waves to a block's keys: by the number of blocks of 128 rows."""
    blocks = batch * heads * -(-length // 128)
    most = 256 if causal else 128
    return ("4x1 many" if blocks > 1024 else "4x1") if blocks > 2 * most else "4x2" if blocks > most else "2x4"


# form of the forward pass and of dq, form of dk and dv; sequences, query heads, key heads, queries, keys; without a mask
FORMS = [
    ("2x4", "2x4", (2, 4, 2, 200, 270), (2, 4, 2, 200, 270)),
    ("4x2", "4x2", (2, 70, 70, 200, 270), (1, 70, 70, 200, 270)),
    ("4x2", "2x4", (3, 60, 20, 140, 140), (1, 66, 22, 140, 140)),
    ("4x1", "4x2", (2, 150, 75, 140, 160), (2, 75, 75, 140, 100)),
    ("4x1", "4x1", (2, 140, 140, 200, 160), (2, 70, 70, 200, 160)),
    ("4x1 many", "4x1", (2, 260, 260, 130, 70), (2, 260, 260, 130, 70)),
]


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("d", [56, 128])
@pytest.mark.parametrize("mask", ["causal", "window", "none"])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: f"{f[0]}-{f[1]}".replace(" ", "-"))
def test_forms(lap, form, mask, d, kind):
    causal = mask != "none"
    b, h, kv, nq, nk = form[2] if causal else form[3]
    window = 37 if mask == "window" else 0
    assert share(b, h, nq, causal) == form[0] and share(b, kv, nk, causal).split()[0] == form[1]
    gen = torch.Generator().manual_seed(d + h)
    q_lens = [nq, nq - 70, 33][:b]
    k_lens = [nk, max(1, nk - 70), 40][:b]
    q, g = rows(gen, b, h, nq, d, kind, q_lens, "bnhd", 1.5), rows(gen, b, h, nq, d, kind, q_lens, "gaps")
    k, v = rows(gen, b, kv, nk, d, kind, k_lens, "bnhd"), rows(gen, b, kv, nk, d, kind, k_lens)
    want = ref.Case(q, k, v, causal=causal, window=window, q_lens=q_lens, k_lens=k_lens)
    args = dict(causal=causal, window=window, q_lens=lens_tensor(q_lens), k_lens=lens_tensor(k_lens))
    got = lap.attention(q, k, v, **args)
    within(got["lse"], want.lse, want.lse_bound, "lse")
    within(got["out"], want.out, want.out_bound, "out")
    grads = lap.attention_grad(g, q, k, v, got["out"], got["lse"], **args)
    for name, (value, bound) in want.grads(g, got["out"]).items():
        within(grads[name], value, bound, name)
    value, bound = want.weights()
    within(lap.attention_weights(q, k, got["lse"], **args)["weights"], value, bound, "weights")


# two waves to a row's keys; keys and rows in parts
@pytest.mark.parametrize("kind,d,heads,kv,n,window", [(BF, 128, 140, 140, 200, 0), (HF, 56, 140, 140, 200, 60), (BF, 64, 2, 1, 1100, 0), (HF, 128, 2, 1, 1100, 0)])
def test_what_is_not_finite(lap, kind, d, heads, kv, n, window):
    ordinary.test_what_is_not_finite_reaches_only_rows_that_see_it(lap, kind, d, heads, kv, n, window)


@pytest.mark.parametrize("kind", [BF, HF])
@pytest.mark.parametrize("scale", [1e-3, 0.06, 1.0])
@pytest.mark.parametrize("heads,kv,n", [(4, 2, 150), (8, 1, 1100)])
def test_scales(lap, heads, kv, n, scale, kind):
    """Every call with a scale of its own."""
    gen = torch.Generator().manual_seed(n)
    d = 64
    q, g = rows(gen, 1, heads, n, d, kind), rows(gen, 1, heads, n, d, kind)
    k, v = rows(gen, 1, kv, n, d, kind), rows(gen, 1, kv, n, d, kind)
    want = ref.Case(q, k, v, causal=True, scale=scale)
    args = dict(causal=True, scale=scale)
    got = lap.attention(q, k, v, **args)
    within(got["out"], want.out, want.out_bound, "out")
    grads = lap.attention_grad(g, q, k, v, got["out"], got["lse"], **args)
    for name, (value, bound) in want.grads(g, got["out"]).items():
        within(grads[name], value, bound, name)
    value, bound = want.weights()
    within(lap.attention_weights(q, k, got["lse"], **args)["weights"], value, bound, "weights")
    step = lap.attention_step(q[:, :, -1], k, v, torch.zeros(1, kv, n, device="cuda"), scale=scale)
    within(step["out"], want.out[:, :, -1], want.out_bound[:, :, -1], "step")
    within(step["lse"], want.lse[:, :, -1], want.lse_bound[:, :, -1], "step's lse")
    last, off = want.p[:, :, -1], (want.p * want.ds)[:, :, -1]
    within(step["weights"], want.shared(last), want.shared(2 * off + 1e-5 * last), "step's weights")
