"""moe_embed and moe_embed_backward against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import step_ends as ends
from training_common import F32, HALF_ULP, TYPES, Context, f64, guarded, randn

pytestmark = pytest.mark.gpu
PAIRS = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")]
TINY = 2.0 ** -126                                             # values below the normal range may be lost


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _wide(t, ld, at=0):
    """The rows of t in rows of ld elements, from element `at` on, and a check that nothing around them was written."""
    whole = torch.full((t.shape[0] + 2, ld), 41.0, dtype=t.dtype, device="cuda")
    inner = whole[1:-1, at:at + t.shape[1]]
    inner.copy_(t)

    def check():
        rest = whole.clone()
        rest[1:-1, at:at + t.shape[1]] = 41.0
        assert (rest == 41.0).all(), "written outside the rows"
    return inner, check


@pytest.mark.parametrize("type,out", PAIRS)
@pytest.mark.parametrize("T,V,d", [(1, 1, 1), (1, 1000, 4096), (3, 7, 5), (64, 50, 8), (33, 9, 1023), (7, 300, 2177), (300, 40, 128), (2, 3, 65536), (5, 4, 7168)])
def test_embed(gpu_lib, T, V, d, type, out):
    rng = np.random.default_rng(T + d)
    ids = rng.integers(0, V, T).astype(np.int32)
    ids[rng.random(T) < 0.2] = rng.choice([-1, V, -2 ** 31, 2 ** 31 - 1])
    table = randn((V, d), type, 1)
    want = ends.embed(ids, f64(table), float(np.float32(d ** 0.5)))
    bound = (F32 + HALF_ULP[out]) * 1.01 * np.abs(want) + TINY  # the product's rounding and the output's
    y, check = guarded((T, d), TYPES[out])
    with Context(gpu_lib, reserve=False) as ctx:
        gpu_lib.moe_embed(ctx, _dev(ids), table.cuda(), d ** 0.5, y)
        check()
        assert (np.abs(f64(y) - want) <= bound).all()
        assert (f64(y)[(ids < 0) | (ids >= V)] == 0).all()
        # rows inside wider ones, at odd places
        for ld, at in ((d + 3, 1), (d + 8, 8), (d + 8, 3)):
            if ld > 65536:
                continue
            src, _ = _wide(table, ld, at)
            dst, around = _wide(torch.zeros((T, d), dtype=TYPES[out]), ld + 4, at)
            gpu_lib.moe_embed(ctx, _dev(ids), src, d ** 0.5, dst)
            around()
            assert torch.equal(dst, y)


def test_embed_keeps_what_the_table_holds(gpu_lib):
    """NaN and infinities of one row reach its tokens and no others; ids of any shape."""
    table = randn((6, 40), "f32", 2)
    table[2, 7], table[4, 0], table[4, 39] = float("nan"), float("inf"), -float("inf")
    ids = torch.tensor([[0, 2, 5], [4, 6, -3]], dtype=torch.int32)
    y = torch.empty((6, 40), device="cuda")
    with Context(gpu_lib, reserve=False) as ctx:
        gpu_lib.moe_embed(ctx, ids.cuda(), table.cuda(), 1.0, y)
        assert torch.equal(y[[0, 2, 3]].cpu(), table[[0, 5, 4]])
        assert (y[4:] == 0).all() and torch.isnan(y[1]).sum() == 1 and torch.equal(y[1, 8:].cpu(), table[2, 8:])
        gpu_lib.moe_embed(ctx, ids[:0].cuda(), table.cuda(), 1.0, torch.empty((0, 40), device="cuda"))


def _text(T, V, load, rng):
    if load == "uniform":
        ids = rng.integers(0, V, T)
    elif load == "zipf":
        p = 1 / (1.0 + np.arange(V))
        ids = rng.permutation(V)[rng.choice(V, T, p=p / p.sum())]
    elif load == "one":
        ids = np.full(T, V // 2)
    elif load == "first_last":
        ids = np.where(np.arange(T) % 2, V - 1, 0)
    elif load == "falling":
        ids = np.arange(T)[::-1] % V
    else:
        ids = np.full(T, -1)
    ids = ids.astype(np.int32)
    if load in ("uniform", "zipf"):
        ids[rng.random(T) < 0.15] = -1
        ids[rng.random(T) < 0.05] = V
    return ids


def _check_gradient(ids, dy, scale, before, accumulate, out, got):
    """fp32 sums of a token's rows in any fixed order, the factor, the sum with what was there, the result's rounding."""
    V, dy = len(before), f64(dy)
    scale = float(np.float32(scale))
    want = ends.embed_backward(dy, ids, scale, before, accumulate)
    size = ends.embed_backward(np.abs(dy), ids, abs(scale), np.abs(before), accumulate)
    terms = np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)[:, None]
    bound = (terms + 3) * F32 * size * 1.01 + HALF_ULP[out] * 1.01 * np.abs(want) + TINY
    assert (np.abs(f64(got) - want) <= bound).all()


@pytest.mark.parametrize("type,out", PAIRS)
@pytest.mark.parametrize("T,V,d,load", [
    (1, 1, 1, "one"), (1, 7, 128, "one"), (2, 5, 9, "one"), (5, 3, 2177, "uniform"), (63, 40, 256, "zipf"), (65, 1000, 31, "uniform"), (777, 500, 1000, "zipf"),
    (1024, 100, 64, "falling"), (1025, 5, 70, "uniform"), (1500, 2, 72, "first_last"), (2048, 3000, 40, "none"), (3000, 17, 128, "one"), (4099, 900, 136, "zipf"),
    (33000, 20000, 16, "zipf"), (40000, 30, 24, "one"), (257, 64, 7168, "zipf"), (9, 3, 65536, "uniform")])
def test_gradient(gpu_lib, T, V, d, load, type, out):
    rng = np.random.default_rng(T + V)
    ids, dy, before = _text(T, V, load, rng), randn((T, d), type, 3), randn((V, d), out, 4, 3.0)
    dy[torch.from_numpy((ids < 0) | (ids >= V))] = float("nan")            # rows that nobody reads
    clean = torch.nan_to_num(dy)
    with Context(gpu_lib) as ctx:
        for accumulate in (False, True):
            g, check = guarded((V, d), TYPES[out])
            again = before.cuda().clone()
            if accumulate:
                g.copy_(before)
            gpu_lib.moe_embed_backward(ctx, dy.cuda(), _dev(ids), 0.75, g, accumulate)
            gpu_lib.moe_embed_backward(ctx, dy.cuda(), _dev(ids), 0.75, again, accumulate)
            check()
            assert torch.equal(g, again)                       # the same bits every time
            _check_gradient(ids, clean, 0.75, f64(before), accumulate, out, g)
            absent = torch.from_numpy(np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V) == 0).cuda()
            assert torch.equal(g[absent], before.cuda()[absent] if accumulate else torch.zeros_like(g[absent]))


@pytest.mark.parametrize("type,out", PAIRS)
@pytest.mark.parametrize("d", [24, 1033])
def test_gradient_of_frequent_tokens(gpu_lib, d, type, out):
    """Tokens whose sorted places go through 31 to 160 runs, some of them from the start of one to the end of another."""
    counts = [8, 31 * 8, 32 * 8, 3, 33 * 8 + 5, 30 * 8 + 1, 8 * 40 - 1, 65 * 8 + 2, 1, 159 * 8 + 7, 64 * 8]
    rng = np.random.default_rng(31)
    ids = rng.permutation(np.repeat(np.arange(len(counts)), counts)).astype(np.int32)
    T, V = len(ids), len(counts) + 1
    dy, before = randn((T, d), type, 32), randn((V, d), out, 33, 3.0)
    with Context(gpu_lib) as ctx:
        for accumulate in (False, True):
            got = []
            for _ in range(3):
                g = before.cuda().clone()
                gpu_lib.moe_embed_backward(ctx, dy.cuda(), _dev(ids), 0.75, g, accumulate)
                got.append(g)
            _check_gradient(ids, dy, 0.75, f64(before), accumulate, out, got[0])
            assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


@pytest.mark.parametrize("T,V,d,load", [(2048, 300, 2560, "zipf"), (2048, 300, 2561, "zipf"), (1025, 300, 5200, "uniform"), (2049, 300, 100, "one")])
def test_gradient_where_the_rows_become_too_wide_for_one_launch(gpu_lib, T, V, d, load):
    rng = np.random.default_rng(d)
    ids, dy, before = _text(T, V, load, rng), randn((T, d), "bf16", 3), randn((V, d), "f32", 4, 3.0)
    with Context(gpu_lib) as ctx:
        for accumulate in (False, True):
            g = before.cuda().clone()
            gpu_lib.moe_embed_backward(ctx, dy.cuda(), _dev(ids), 0.75, g, accumulate)
            _check_gradient(ids, dy, 0.75, f64(before), accumulate, "f32", g)


@pytest.mark.parametrize("type,out", PAIRS)
def test_gradient_of_strided_rows(gpu_lib, type, out):
    rng = np.random.default_rng(5)
    T, V, d = 700, 90, 203
    ids, dy, before = _dev(_text(T, V, "zipf", rng)), randn((T, d), type, 6).cuda(), randn((V, d), out, 7).cuda()
    with Context(gpu_lib) as ctx:
        for accumulate in (False, True):
            want = before.clone()
            gpu_lib.moe_embed_backward(ctx, dy, ids, 2.0, want, accumulate)
            for ld, at in ((205, 1), (211, 3), (216, 8)):
                src, _ = _wide(dy, ld, at)
                dst, check = _wide(before, ld + 2, at)
                gpu_lib.moe_embed_backward(ctx, src, ids, 2.0, dst, accumulate)
                check()
                assert torch.equal(dst, want)


def test_gradient_of_no_tokens(gpu_lib):
    g = torch.full((5, 12), 9.0, device="cuda")
    none, ids = torch.empty((0, 12), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_embed_backward(ctx, none, ids, 1.0, g, True)
        assert (g == 9).all()
        gpu_lib.moe_embed_backward(ctx, none, ids, 1.0, g)
        assert (g == 0).all()
    with Context(gpu_lib, reserve=False) as ctx, pytest.raises(gpu_lib.MoEError):
        gpu_lib.moe_embed_backward(ctx, none, ids, 1.0, g)


def test_gradient_is_that_of_the_lookup(gpu_lib):
    """<dy, embed(table + h v) - embed(table - h v)> / 2h, which is linear in the table: the gradient's product with v, up to fp32's roundings."""
    g = torch.Generator(device="cuda").manual_seed(8)
    T, V, d = 500, 64, 96
    ids = torch.randint(-1, V + 1, (T,), generator=g, device="cuda", dtype=torch.int32)
    table, v = torch.randn((V, d), generator=g, device="cuda"), torch.randn((V, d), generator=g, device="cuda")
    dy, grad = torch.randn((T, d), generator=g, device="cuda"), torch.empty((V, d), device="cuda")
    up, down = torch.empty_like(dy), torch.empty_like(dy)
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_embed(ctx, ids, table + 0.5 * v, 3.0, up)
        gpu_lib.moe_embed(ctx, ids, table - 0.5 * v, 3.0, down)
        gpu_lib.moe_embed_backward(ctx, dy, ids, 3.0, grad)
    slope = ((up.double() - down.double()) * dy.double()).sum()
    size = (dy.double().abs() * (up.double().abs() + down.double().abs())).sum() + (grad.double().abs() * v.double().abs()).sum()
    # table +- v/2 and the products: a rounding each of `up` and `down`; a token's sum: at most T of them
    assert (slope - (grad.double() * v.double()).sum()).abs() <= 4 * F32 * size + T * F32 * (grad.double().abs() * v.double().abs()).sum()
