"""The balance in one workgroup and in three launches, on both sides of the limit between them: one workgroup takes no more than
16 logits a lane, or all tokens at once, so that many tokens with few experts do not wait for one another."""
import pytest
import torch

from loss_reference import Balance

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
# tokens, experts, slots, type, whether one workgroup takes it: 16 wavefronts of 64 lanes, 16 bytes of a token a lane (more from 65 experts on in
# binary32, from 129 in bf16), lanes a power of two
ROUTES = [(4096, 1, 1, F32, True), (4097, 1, 1, F32, False), (16384, 1, 1, F32, False), (2048, 1, 1, BF16, True), (2049, 1, 1, BF16, False),
          (8192, 2, 1, BF16, False), (1024, 9, 2, F32, True), (1025, 9, 2, F32, False), (1024, 9, 2, BF16, True), (1820, 9, 2, BF16, False),
          (963, 17, 2, F32, False), (256, 33, 2, BF16, True), (496, 33, 2, BF16, False), (512, 32, 4, F32, True), (513, 32, 4, F32, False),
          (64, 8, 2, F32, True), (16, 1024, 8, F32, True), (17, 1024, 8, F32, False), (16, 1024, 8, BF16, True), (17, 1024, 8, BF16, False)]


@pytest.mark.parametrize("tokens,experts,slots,kind,one", ROUTES, ids=str)
def test_route_and_results(gpu_lib, tokens, experts, slots, kind, one):
    from paper_1901_01544_amd import losses
    gen = torch.Generator(device=DEV).manual_seed(tokens + experts)
    x = (2.0 * torch.randn(tokens, experts, generator=gen, device=DEV)).to(kind)
    chosen = torch.randint(-1, experts + 1, (tokens, slots), generator=gen, device=DEV, dtype=torch.int32)
    keep = (torch.rand(tokens, generator=gen, device=DEV) < 0.8).to(torch.uint8)
    loss, counts = torch.empty(2, device=DEV), torch.empty(experts, dtype=torch.int32, device=DEV)
    dx = torch.full_like(x, float("nan"))
    ws = torch.full((losses.balance_workspace_bytes(tokens, experts),), 0xFF, dtype=torch.uint8, device=DEV)
    launches = {}
    for name in ("k_balance_one", "k_balance_rows"):
        gpu_lib.timing_enable(name, 4)
        losses.balance(x, chosen, loss, counts, dx, ws, balance=0.5, z=0.25, keep=keep)
        torch.cuda.synchronize()
        launches[name] = gpu_lib.timing_collect()[1]
    assert launches == {"k_balance_one": int(one), "k_balance_rows": int(not one)}
    Balance(x, chosen, 0.5, 0.25, keep).check(loss, counts, dx)
