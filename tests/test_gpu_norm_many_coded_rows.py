"""moe_add_rmsnorm with codes on more rows than one launch takes: 16 rows to a block of 64 threads, from 2^29 rows on."""
import gc

import pytest
import torch

from training_common import Context

pytestmark = pytest.mark.gpu
ROWS, COLS, TILE = 2 ** 29 + 5, 128, 4096


def test_codes_of_very_many_rows(gpu_lib):
    gc.collect()
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 225 * 10 ** 9:
        pytest.skip("needs 209 GB of the GPU's memory for itself")
    tile = torch.randn((TILE, COLS), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    n = ROWS // TILE
    x = torch.empty((ROWS, COLS), dtype=torch.bfloat16, device="cuda")
    x[:n * TILE].view(n, TILE, COLS).copy_(tile.expand(n, TILE, COLS))
    x[n * TILE:] = tile[:ROWS - n * TILE]
    q, s = torch.empty((ROWS, COLS), dtype=torch.uint8, device="cuda"), torch.full((1, ROWS), 9.0, device="cuda")
    tq, ts = torch.empty((TILE, COLS), dtype=torch.uint8, device="cuda"), torch.empty((1, TILE), device="cuda")
    gain = torch.ones(COLS, device="cuda")
    try:
        with Context(gpu_lib, reserve=False) as ctx:
            gpu_lib.moe_add_rmsnorm(ctx, tile, None, gain, 1e-6, q=tq, scales=ts)
            gpu_lib.moe_add_rmsnorm(ctx, x, None, gain, 1e-6, q=q, scales=s)
        for i in range(0, n, 4096):
            m = min(4096, n - i)
            at = slice(i * TILE, (i + m) * TILE)
            assert (q[at].view(m, TILE, COLS) == tq).all() and (s[0, at].view(m, TILE) == ts[0]).all()
        left = ROWS - n * TILE
        assert torch.equal(q[n * TILE:], tq[:left]) and torch.equal(s[0, n * TILE:], ts[0, :left])
    finally:
        del x, q, s
        torch.cuda.empty_cache()
