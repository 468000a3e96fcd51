"""Refusals of the calls at the two ends of a policy step, before anything touches a device."""
import ctypes

import pytest
import torch

import paper_2512_07710_amd as moe

N, P, Q = None, 1 << 20, 1 << 21                               # pointers: none, and two that nobody follows


@pytest.fixture(scope="module")
def call():
    """call(name, *arguments): the status.  The context is memory that looks like one with a workspace, and without a GPU nothing can be launched."""
    if torch.cuda.is_available():
        pytest.skip("for machines without a GPU: a call that is not refused would run on made-up pointers")
    lib, ctx = moe.load_library(), ctypes.create_string_buffer(b"\x40" * 4096, 4096)

    def status(name, *a):
        return getattr(lib, name)(ctypes.addressof(ctx), *a)
    return status


def _changed(base, changes):
    for at, values in changes.items():
        for v in values:
            yield [v if i == at else b for i, b in enumerate(base)], (at, v)


FLOATS = (float("nan"), float("inf"), float("-inf"))


def test_without_a_context():
    lib = moe.load_library()
    one = (ctypes.c_int64 * 1)(1)
    assert lib.moe_embed(N, P, 1, P, 10, 8, 8, 0, 1.0, P, 8, 0) == -1
    assert lib.moe_embed_backward(N, P, P, 1, 10, 8, 8, 0, 1.0, 0, P, 8, 0) == -1
    assert lib.moe_token_logp(N, P, 8, 0, 1, 8, P, 1, 1.0, P, P, 0, N, N, N) == -1
    assert lib.moe_token_logp_backward(N, P, 8, 0, 1, 8, P, 1, 1.0, P, N, P, N, Q, 8, 0) == -1
    assert lib.moe_grad_norm(N, one, one, (ctypes.c_int32 * 1)(0), 1, P, N) == -1
    assert lib.moe_clip_grads(N, one, one, (ctypes.c_int32 * 1)(0), 1, P, 1.0, N) == -1


def test_embed(call):
    #       ids T  table V  d  ld dt scale y ld_y out
    base = [P, 4, P, 10, 8, 8, 0, 1.0, Q, 8, 0]
    bad = {0: [N, P + 1], 1: [-1, 2 ** 30 + 1], 2: [N, P + 1], 3: [0, -1], 4: [0, -8, 9, 65537], 5: [7, 0, 2 ** 31], 6: [2, -1], 7: FLOATS, 8: [N, Q + 1],
           9: [7, 2 ** 31], 10: [2, -1]}
    for args, what in _changed(base, bad):
        assert call("moe_embed", *args) == -1, what
    assert call("moe_embed", P, 4, P + 2, 10, 8, 8, 1, 1.0, Q, 8, 0) == -1     # inside an element
    assert call("moe_embed", N, 0, N, 10, 8, 8, 0, 1.0, N, 8, 0) == 0          # no tokens


def test_embed_backward(call):
    #       dy ids T  V  d  ld dt scale acc dtable ld_grad grad
    base = [P, P, 4, 10, 8, 8, 0, 1.0, 0, Q, 8, 0]
    bad = {0: [N, P + 1], 1: [N, P + 2], 2: [-1, 2 ** 21 + 1], 3: [0, -1], 4: [0, 9, 65537], 5: [7, 2 ** 31], 6: [2, -1], 7: FLOATS, 9: [N, Q + 1],
           10: [7, 2 ** 31], 11: [2, -1]}
    for args, what in _changed(base, bad):
        assert call("moe_embed_backward", *args) == -1, what
    assert call("moe_embed_backward", P, P, 4, 10, 8, 8, 0, 1.0, 0, Q + 2, 8, 1) == -1


def test_token_logp(call):
    #       logits ld dt rows V ids m temp logp entropy n top_idx top_logp stats
    base = [P, 8, 0, 4, 8, P, 2, 1.0, P, P, 3, P, P, P]
    bad = {0: [N, P + 1], 1: [7, 2 ** 31], 2: [2, -1], 3: [-1, 2 ** 30 + 1], 4: [0, -1, 9], 5: [N, P + 2], 6: [-1, 65], 7: (0.0, -1.0, 1e-45, 2e6, *FLOATS),
           8: [N, P + 1], 9: [P + 1], 10: [-1, 65], 11: [N, P + 2], 12: [N, P + 2], 13: [P + 2]}
    for args, what in _changed(base, bad):
        assert call("moe_token_logp", *args) == -1, what
    assert call("moe_token_logp", P, 8, 0, 4, 8, N, 0, 1.0, N, N, 0, N, N, N) == -1        # nothing asked for
    assert call("moe_token_logp", N, 8, 0, 0, 8, N, 2, 1.0, N, N, 3, N, N, N) == 0         # no rows


def test_token_logp_backward(call):
    #       logits ld dt rows V ids m temp dlogp dentropy stats entropy dlogits ld_grad grad
    base = [P, 8, 0, 4, 8, P, 2, 1.0, P, P, P, P, Q, 8, 0]
    bad = {0: [N, P + 1], 1: [7, 2 ** 31], 2: [2], 3: [-1, 2 ** 30 + 1], 4: [0, 9], 5: [N, P + 2], 6: [-1, 65], 7: (0.0, 1e-7, 2e6, *FLOATS), 8: [N, P + 2],
           9: [P + 2], 10: [N, P + 2], 11: [N, P + 2], 12: [N, Q + 1], 13: [7, 2 ** 31], 14: [2, -1]}
    for args, what in _changed(base, bad):
        assert call("moe_token_logp_backward", *args) == -1, what
    in_place = list(base)
    in_place[12] = P
    for at, v in ((13, 9), (14, 1)):                           # in the place of logits of another stride or type
        assert call("moe_token_logp_backward", *[v if i == at else b for i, b in enumerate(in_place)]) == -1
    assert call("moe_token_logp_backward", N, 8, 0, 0, 8, N, 2, 1.0, N, N, N, N, N, 8, 0) == 0


def _arrays(*of):
    types = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32)
    return [(t * len(v))(*v) for t, v in zip(types, of)]


def test_lists(call):
    good = ([P, N, Q], [10, 0, 5], [0, 0, 1])
    bad = [([P, N, N], [10, 0, 5], [0, 0, 1]), ([P + 1, N, Q], [10, 0, 5], [0, 0, 1]), ([P, N, Q + 2], [10, 0, 5], [0, 0, 1]), ([P, N, Q], [10, -1, 5], [0, 0, 1]),
           ([P, N, Q], [10, 0, 5], [0, 0, 2]), ([P, P, Q], [2 ** 40, 1, 5], [0, 0, 1])]
    for lists in bad:
        assert call("moe_grad_norm", *_arrays(*lists), 3, P, N) == -1
        assert call("moe_clip_grads", *_arrays(*lists), 3, P, 1.0, N) == -1
    a, c, t = _arrays(*good)
    for lists in bad[:3]:
        assert call("moe_clip_grads", a, c, t, 3, P, 1.0, _arrays(*lists)[0]) == -1
    for args in ((N, c, t, 3), (a, N, t, 3), (a, c, N, 3), (a, c, t, -1), (a, c, t, 65537)):
        assert call("moe_grad_norm", *args, P, N) == -1
        assert call("moe_clip_grads", *args, P, 1.0, N) == -1
    for sum_sq in (N, P + 4):
        assert call("moe_grad_norm", a, c, t, 3, sum_sq, N) == -1
        assert call("moe_clip_grads", a, c, t, 3, sum_sq, 1.0, N) == -1
    assert call("moe_grad_norm", a, c, t, 3, P, P + 2) == -1
    for max_norm in (-1.0, *FLOATS):
        assert call("moe_clip_grads", a, c, t, 3, P, max_norm, N) == -1
    for shifted in ([P + 2, N, Q], [P, N, Q - 16], [P - 18, N, Q]):
        assert call("moe_clip_grads", a, c, t, 3, P, 1.0, _arrays(shifted, *good[1:])[0]) == -1
    assert call("moe_clip_grads", N, N, N, 0, P, 1.0, N) == 0


def test_what_the_binding_refuses():
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    with pytest.raises(moe.MoEError):
        moe.GradList([t(4)])                                   # not on a GPU
    with pytest.raises(moe.MoEError):
        moe.moe_embed(None, t(4, dtype=torch.int32), t(10, 8), 1.0, t(4, 8))
    with pytest.raises(moe.MoEError):
        moe.moe_embed(None, t(4, dtype=torch.int32), t(10, 8, dtype=torch.float16), 1.0, t(4, 8))
    with pytest.raises(moe.MoEError):
        moe.moe_token_logp(None, t(4, 8), t(4, dtype=torch.int32), t(4))
