"""Edges of the real-valued operators on the GPU."""
import threading

import pytest
import torch

import real_reference as ref
from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def normal(seed, *shape, dtype=BF, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=g).to(dtype)


@pytest.mark.parametrize("M,N,K", [(64, 1011, 512), (512, 1010, 1024), (3, 9, 8)])
@pytest.mark.parametrize("bias", (True, False), ids=("bias", "plain"))
def test_linear_backward_in_the_workspace_asked_for(ctx, M, N, K, bias):
    """x and W in whole 16-byte groups, contiguous dy not: a layer without activation copies dy."""
    x, W, dy = normal(1, M, K), normal(2, N, K, scale=K ** -0.5), normal(3, M, N)
    b = normal(4, N) if bias else None
    layer = ctx.make_linear(W, b)
    n = ctx.linear_workspace_bytes(layer, x, backward=True)
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:n] if n else None)
    want = ref.linear(x, W, b, None, "none", dy)
    for key, t in zip(("dx", "dW", "db"), ctx.linear_backward(layer, dy, x)):
        if t is not None:
            ref.check(t, *want[key], key)
    ctx.device_status()
    assert (ws[n:] == 0x7F).all(), "written beyond the workspace"
    ctx.set_workspace(None)


def test_contexts_of_two_threads_at_different_widths():
    """A context per host thread is allowed: what one thread's launches need must not depend on the other's.  Both widths run the same
    kernel with different amounts of shared memory."""
    widths, failures, results = (2048, 4096), [], {}

    def steps(D, start):
        try:
            stream = torch.cuda.Stream()
            c = binding.Context(0, stream)
            with torch.cuda.stream(stream):
                x, b, ds, dn, w = (normal(k, 4, D) for k in range(5))
                layer = c.make_block_norm(D, BF, kind="layer", post=True, pre_weight=w[0])
                ws = torch.empty(c.block_norm_workspace_bytes(layer, 4), dtype=torch.uint8, device="cuda")
                c.set_workspace(ws)
                stats = c.empty(4, 4, dtype=FF)
                c.block_norm(layer, x, b, stats=stats)
                start.wait()
                for _ in range(3000):
                    results[D] = c.block_norm_backward(layer, ds, dn, x, b, stats)["dblock"]
            stream.synchronize()
            c.close()
        except Exception as e:                    # raised in the test's own thread below
            failures.append(e)

    build.build()
    start = threading.Barrier(len(widths), timeout=60)
    threads = [threading.Thread(target=steps, args=(D, start)) for D in widths]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    for D in widths:
        x, b, ds, dn, w = (normal(k, 4, D) for k in range(5))
        par = {"kind": "layer", "eps": 1e-6, "alpha": 1.0, "post": True, "pre": True, "pre_weight": w[0]}
        ref.check(results[D], *ref.block_norm(x, b, par, ds, dn)["dblock"], "dblock")
