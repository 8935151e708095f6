"""Products of few rows split their sums over a cluster.  Where a wait of one of its CTAs runs out, none of them writes outputs that lack its share: they stay as they were, the
call reports the failure, and the next one is right."""
import pytest
import torch

from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, FF = torch.bfloat16, torch.float32


@pytest.mark.parametrize("M,N,K", [(1, 256, 8192), (5, 300, 4096), (40, 1000, 4096), (100, 128, 8200)])
def test_no_output_lacks_a_share(M, N, K):
    build.build()
    c = binding.Context(0)
    g = torch.Generator(device="cuda").manual_seed(M)
    mk = lambda *s: torch.randn(*s, device="cuda", generator=g).to(BF)  # noqa: E731
    x, W, U = mk(M, K), mk(N, K), mk(N, K)
    q, w, u = c.mx_quantize(x), c.mx_quantize(W, "e2m1"), c.mx_quantize(U, "e2m1")
    dense, glu, dense16, glu16 = c.make_mx_linear(w), c.make_mx_gated(w, u), c.make_linear(W), c.make_gated(W, U)
    ws = torch.empty(max(256, c.linear_workspace_bytes(dense16, x), c.gated_workspace_bytes(glu16, x)), dtype=torch.uint8, device="cuda")
    c.set_workspace(ws)
    y, pre, y_mx = torch.empty(M, N, dtype=BF, device="cuda"), torch.empty(2, M, N, device="cuda"), c.make_mx(M, N)
    calls = [lambda: c.mx_linear(dense, q, out=y, pre=pre[0]), lambda: c.mx_gated(glu, q, out=y, pre=pre), lambda: c.linear(dense16, x, out=y, pre=pre[0]),
             lambda: c.gated(glu16, x, out=y, pre=pre), lambda: c.mx_linear(dense, q, out=y_mx), lambda: c.mx_gated(glu, q, out=y_mx)]

    def fill():
        y.fill_(77.0), pre.fill_(77.0), y_mx.values.fill_(0xA5), y_mx.scales.fill_(0xA5)

    for call in calls:
        fill()
        call()
        want = [t.clone() for t in (y, pre, y_mx.values)]
        fill()
        c.set_wait_limit_ns(5_000_000)
        c.debug_drop_loads(2)
        call()
        with pytest.raises(binding.BnnError):
            c.device_status()
        c.debug_drop_loads(0)
        c.set_wait_limit_ns(2_000_000_000)
        assert (y == 77).all() and (pre == 77).all(), "an output without a CTA's share"
        assert (y_mx.values == 0xA5).all() and (y_mx.scales == 0xA5).all(), "a microscaled output without a CTA's share"
        call()
        c.device_status()
        assert all(torch.equal(a, b) for a, b in zip((y, pre, y_mx.values), want))
    c.set_workspace(None)
    c.close()
