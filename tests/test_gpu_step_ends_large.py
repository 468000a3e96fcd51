"""Arrays of more than 2^32 elements, batches of very many tokens and gradients: what lies behind them is read and written where it belongs."""
import pytest
import torch

from training_common import F32, HALF_ULP, Context

pytestmark = pytest.mark.gpu
BF16, CUDA = torch.bfloat16, "cuda"


@pytest.fixture(autouse=True)
def _empty_cache():
    yield
    torch.cuda.empty_cache()


def test_embedding_of_a_table_past_32_bits(gpu_lib):
    V, d, T = 700000, 7168, 3000                               # 5.0e9 elements
    table = torch.empty((V, d), dtype=BF16, device=CUDA)
    ids = torch.randint(0, V, (T,), device=CUDA, dtype=torch.int32)
    ids[:3] = torch.tensor([V - 1, 0, V - 1], dtype=torch.int32)
    table[ids.long()] = torch.randn((T, d), device=CUDA).to(BF16)
    y = torch.empty((T, d), dtype=BF16, device=CUDA)
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_embed(ctx, ids, table, 2.0, y)
        assert torch.equal(y, table[ids.long()] * 2)
        gpu_lib.moe_embed_backward(ctx, y, ids, 0.5, table)
        at, place = torch.unique(ids, return_inverse=True)
        want = torch.zeros((len(at), d), device=CUDA, dtype=torch.float64).index_add_(0, place, y.double() * 0.5)
        assert ((table[at.long()].double() - want).abs() <= (HALF_ULP["bf16"] + 8 * F32) * 1.01 * want.abs() + 1e-5 * F32).all()
        seen = torch.zeros(V, dtype=torch.bool, device=CUDA)
        seen[at.long()] = True
        for i in range(0, V, 100000):
            assert not (table[i:i + 100000].abs().amax(dim=1) > 0)[~seen[i:i + 100000]].any()


@pytest.mark.parametrize("T,V,d", [(2 ** 21, 50000, 8), (140000, 200, 24), (700000, 3, 7168)])
def test_gradient_of_very_many_tokens(gpu_lib, T, V, d):
    """Runs merged more than once; a few tokens over very many runs.  700000 x 7168 is past 2^32."""
    g = torch.Generator(device=CUDA).manual_seed(T)
    ids = torch.randint(-1, V, (T,), generator=g, device=CUDA, dtype=torch.int32)
    dy = torch.randint(-8, 9, (T, d), generator=g, device=CUDA, dtype=torch.int8).to(BF16)  # whole numbers: sums of up to 2^24 are exact
    dtable = torch.full((V, d), 5.0, device=CUDA)
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_embed_backward(ctx, dy, ids, 1.0, dtable)
        want = torch.zeros((V + 1, d), device=CUDA, dtype=torch.float64)
        for i in range(0, T, 1 << 16):
            want.index_add_(0, ids[i:i + (1 << 16)].long() + 1, dy[i:i + (1 << 16)].double())
        assert torch.equal(dtable.double(), want[1:])


def test_log_probabilities(gpu_lib):
    rows, V, last = 33000, 131072, 600
    z = torch.empty((rows, V), dtype=BF16, device=CUDA).normal_()
    ids = torch.randint(0, V, (rows, 2), device=CUDA, dtype=torch.int32)
    new = lambda n: [torch.empty((n, 2), device=CUDA), torch.empty(n, device=CUDA), torch.empty((n, 9), dtype=torch.int32, device=CUDA),  # noqa: E731
                     torch.empty((n, 9), device=CUDA), torch.empty((n, 2), device=CUDA)]
    out, short, at = new(rows), new(last), slice(rows - last, rows)
    tail = z[at].clone()
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_token_logp(ctx, z, ids, *out)
        gpu_lib.moe_token_logp(ctx, tail, ids[at], *short)
        # (600 rows in blocks of another size: the sums' roundings differ)
        assert torch.equal(out[2][at], short[2])
        for a, b in zip(out, short):
            if a is not out[2]:
                assert ((a[at].double() - b.double()).abs() <= 64 * F32 * (1 + b.double().abs())).all()
        exact = torch.log_softmax(tail.double(), dim=1).gather(1, ids[at].long())
        assert ((out[0][at].double() - exact).abs() <= 128 * F32 * (1 + exact.abs())).all()
        d, grad = torch.randn((rows, 2), device=CUDA), torch.empty_like(tail)
        gpu_lib.moe_token_logp_backward(ctx, z, ids, d, None, out[4], None, z)             # in place
        gpu_lib.moe_token_logp_backward(ctx, tail, ids[at], d[at], None, out[4][at], None, grad)
        assert torch.equal(z[at], grad)


def test_very_many_short_rows(gpu_lib):
    n, few = 2 ** 26 + 5, 1024                                 # times 64 threads: past 2^32
    tile = lambda t: t.repeat(n // few + 1, *[1] * (t.dim() - 1))[:n].contiguous()  # noqa: E731
    z, ids = tile(torch.randn((few, 2), device=CUDA)), tile((torch.arange(few, device=CUDA) % 2).to(torch.int32))
    logp, top, lp = torch.full((n,), 9.0, device=CUDA), torch.full((n, 1), 9, dtype=torch.int32, device=CUDA), torch.full((n, 1), 9.0, device=CUDA)
    with Context(gpu_lib) as ctx:
        gpu_lib.moe_token_logp(ctx, z, ids, logp, None, top, lp)
    exact = torch.log_softmax(z[:few].double(), dim=1)
    assert ((logp[:few].double() - exact.gather(1, ids[:few, None].long())[:, 0]).abs() <= 16 * F32 * (1 + exact.abs().amax())).all()
    assert torch.equal(top[:few, 0].long(), z[:few].argmax(dim=1))
    whole = n // few * few
    for a in (logp, top[:, 0], lp[:, 0]):
        assert (a[:whole].view(-1, few) == a[:few]).all() and torch.equal(a[whole:], a[:n - whole])


def test_norm_and_clipping(gpu_lib):
    n = 2 ** 32 + 12345
    big, small = torch.empty(n, dtype=BF16, device=CUDA), [torch.ones(3, device=CUDA) for _ in range(5000)]
    big.fill_(0.5)
    big[-1] = 3.0
    s, norm = torch.empty(1, dtype=torch.float64, device=CUDA), torch.empty(1, device=CUDA)
    with Context(gpu_lib) as ctx:
        grads = gpu_lib.GradList([*small, big, torch.ones(1, device=CUDA)])
        gpu_lib.moe_grad_norm(ctx, grads, s, norm)
        assert float(s) == 0.25 * (n - 1) + 9 + 15000 + 1      # (exact in fp64)
        gpu_lib.moe_clip_grads(ctx, grads, s, float(s) ** 0.5 / 2)
    assert big[-1] == 1.5 and torch.equal(small[4999], torch.full((3,), 0.5, device=CUDA)) and grads.tensors[-1][0] == 0.5
    for i in range(0, n - 1, 1 << 30):
        assert (big[i:min(i + (1 << 30), n - 1)] == 0.25).all()
