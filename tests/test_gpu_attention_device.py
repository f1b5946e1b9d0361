"""Calls go to their tensors' GPU, also while another one is the current one (which this test only pretends)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_every_call_makes_its_tensors_gpu_the_current_one(monkeypatch):
    import paper_1903_06631_amd as lap
    from paper_1903_06631_amd import attention_ops as ops
    lap.load_library()
    entered = []

    class Recorded(torch.cuda.device):
        def __enter__(self):
            entered.append(self.idx)
            return super().__enter__()

    q, k = torch.randn(1, 4, 9, 64, device="cuda").half(), torch.randn(1, 2, 20, 64, device="cuda").half()
    w, pos = torch.rand(1, 2, 20, device="cuda"), torch.arange(20, dtype=torch.int32, device="cuda").expand(1, 2, 20).contiguous()
    at = torch.tensor([20], dtype=torch.int32, device="cuda")

    def calls():
        f = lap.attention(q, k, k)
        return [f["out"], f["lse"], *lap.attention_grad(q, q, k, k, f["out"], f["lse"]).values(), lap.attention_weights(q, k, f["lse"])["weights"],
                lap.attention_step(q[:, :, 0], k, k)["out"], *lap.cache_evict(k, k, w, 5, 2).values(),
                lap.cache_insert(k[:, :, 0], k[:, :, 0], k.clone(), k.clone(), w.clone(), pos.clone(), at, 2)["slots"]]

    want = calls()
    monkeypatch.setattr(torch.cuda, "device", Recorded)
    monkeypatch.setattr(ops, "_device", lambda: 0)
    calls()
    assert entered == []
    monkeypatch.setattr(ops, "_device", lambda: 1)
    got = calls()
    assert entered == [0] * 6 and all(torch.equal(a, b) for a, b in zip(want, got))
