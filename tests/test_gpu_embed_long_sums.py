"""moe_embed_backward where one token has so many rows that adding them up one after another would lose digits."""
import pytest
import torch

from training_common import F32, TYPES, Context

pytestmark = pytest.mark.gpu
CUDA = "cuda"
# Additions one after another that a row's share of the sum goes through at these sizes (the rule's own host test has the number), the factor, the sum with what is there
CHAIN = 200 + 2


def _rows(T, d, type, how):
    if how == "even":                          # of one sign and size, other in each column: each addition's error has the sign of the one before
        column = torch.linspace(0.05, 1.0, d, device=CUDA).to(TYPES[type])
        return column.expand(T, d).contiguous()
    dy = torch.full((T, d), 2.0 ** -12 * 0.96875, dtype=TYPES[type], device=CUDA)              # less than half a last place of 4096
    dy[::1024] = 4096.0
    return dy


@pytest.mark.parametrize("how", ["even", "one large"])
@pytest.mark.parametrize("T,d,type", [(2 ** 21, 64, "f32"), (2 ** 21, 64, "bf16"), (2 ** 20, 512, "f32"), (2 ** 20 + 77, 131, "bf16")])
def test_sums_of_a_frequent_token(gpu_lib, T, d, type, how):
    dy = _rows(T, d, type, how)
    ids = torch.full((T,), 1, dtype=torch.int32, device=CUDA)
    ids[3::9973] = 2                           # (a few rows of another token, and of none)
    ids[5::9967] = -1
    before = torch.full((4, d), 3.0, device=CUDA)
    want = torch.zeros((4, d), dtype=torch.float64, device=CUDA)
    for v in (1, 2):
        of = dy[ids == v]
        for i in range(0, len(of), 1 << 18):
            want[v] += 0.75 * of[i:i + (1 << 18)].double().sum(dim=0)
    with Context(gpu_lib) as ctx:
        for accumulate in (False, True):
            g = before.clone()
            gpu_lib.moe_embed_backward(ctx, dy, ids, 0.75, g, accumulate)
            exact = want + before.double() if accumulate else want
            error = (g.double() - exact).abs() / exact.clamp(min=1e-30)
            assert (error <= CHAIN * F32).all(), float(error.max() / F32)
