"""The products' sums are held in 32 bits whichever way a call is dealt: bounds that operands or partial sums in fewer bits do
not meet (sum_error.py derives them)."""
import pytest
import torch

from paper_2502_06282_b200 import binding as jk
from tests.sum_error import fma_bound, off, tensor_bound
from tests.test_gpu_layer import make_ctx, torch_mx8

pytestmark = pytest.mark.gpu


def check(ctx, R, N, K, bound, pack, gated=False):
    """Outputs in f32.  Gated blocks: once with a second factor of 1, once with a first one."""
    g = torch.Generator(device="cuda").manual_seed(R + N + K)
    (xd, x), (wd, w) = pack(torch.randn(R, K, generator=g, device="cuda")), pack(torch.randn(N, K, generator=g, device="cuda") * 0.05)
    exact = x @ w.T
    ops = [jk.Linear(ctx, wd)]
    if gated:
        zero, one = pack(torch.zeros(N, K, device="cuda"))[0], torch.ones(N, dtype=ctx.tdtype, device="cuda")
        ops = [jk.Linear(ctx, wd, w_up=zero, bias_up=one), jk.Linear(ctx, zero, bias=one, w_up=wd)]
    for op in ops:
        y = torch.full((R, N), float("nan"), device="cuda")
        ctx.linear(op, xd, y)
        rms, top = off(y.double(), exact, x, w)
        assert rms <= bound and top <= 8 * bound, (rms / bound, top / bound)
    assert ctx.read_status() == 0


# clusters; even shares whose tiles span CTAs; whole tiles; many rows, whole and cut
@pytest.mark.parametrize("kind", ["T", "mx8"])
@pytest.mark.parametrize("R,N,K,gated", [
    (60, 4096, 4096, False), (60, 640, 4096, False), (17, 5120, 4096, False), (250, 9000, 4096, False), (128, 11008, 8192, False),
    (1, 32000, 1024, False), (60, 2048, 4096, True), (128, 11008, 4096, True), (300, 2048, 8192, False), (700, 5119, 2048, False),
    (257, 9000, 8192, False), (1100, 2000, 8192, False), (256, 5120, 13824, False), (1100, 1200, 8192, True), (480, 4864, 4096, True),
    (4099, 1376, 512, False)])
def test_sums_of_the_tensor_cores(R, N, K, gated, kind):
    pack = torch_mx8 if kind == "mx8" else (lambda x: (x.bfloat16(), x.bfloat16().double()))
    check(make_ctx("bf16"), R, N, K, tensor_bound(K, 16 if kind == "T" else 32), pack, gated)


# warps of one and two outputs; blocks of 32, of 64 (alone and shared) and of 128 rows
@pytest.mark.parametrize("R,N,K,gated", [(1, 2373, 4096, False), (16, 4097, 2048, False), (5, 1190, 2048, True), (20, 512, 4096, False),
                                         (64, 512, 4096, False), (64, 512, 2048, True), (256, 4096, 1024, False), (1024, 1300, 2048, False)])
def test_sums_in_f32(R, N, K, gated):
    check(make_ctx("f32"), R, N, K, fma_bound(K), lambda x: (x, x.double()), gated)


@pytest.mark.parametrize("R", [3, 40, 300])
def test_sums_without_the_tensor_path(R):
    for kind, pack in (("T", lambda x: (x.bfloat16(), x.bfloat16().double())), ("mx8", torch_mx8)):
        ctx = make_ctx("bf16")
        ctx.set_tensor_path(False)
        check(ctx, R, 520, 2048, fma_bound(2048), pack)
