"""What the router's results hold on to: their own memory, not the scratch of the call that made them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,e,k", [(30011, 128, 8), (2000, 1024, 4), (37, 8, 2), (160000, 5, 1)])
def test_results_hold_no_scratch(t, e, k):
    from paper_2508_15706_b200 import inner
    x = torch.randn(t, e, device="cuda")
    r = inner.route_forward(x, k)
    own = sum((y.numel() * y.element_size() + 255) // 256 * 256 for y in r)
    # small scratch may lie with them: 16 KB at most
    assert all(y.untyped_storage().nbytes() <= own + 16384 for y in r), (r.weights.untyped_storage().nbytes(), own)
    torch.cuda.synchronize()
    asked = lambda: torch.cuda.memory_stats()["requested_bytes.all.current"]  # (not what the allocator's blocks have beyond that)
    before = asked()
    held = [inner.route_forward(x, k) for _ in range(4)]
    torch.cuda.synchronize()
    assert asked() - before <= 4 * (own + 16384 + 512)
    for again in held:
        assert all(torch.equal(a, b) for a, b in zip(again, r))
