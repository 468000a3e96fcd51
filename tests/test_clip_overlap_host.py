"""moe_clip_grads refuses outputs that lie over gradients other than their own: blocks would overwrite what others have not read yet."""
import ctypes
import random

import pytest
import torch

import paper_2512_07710_amd as moe

BASE = 1 << 30                                                 # addresses that nobody follows
REFUSED, PASSED_ON = -1, -2                                    # (without a GPU no launch succeeds)


@pytest.fixture(scope="module")
def clip():
    """clip(places of the gradients, of the outputs, elements, types): the status.  The context is memory that looks like one with a workspace."""
    if torch.cuda.is_available():
        pytest.skip("for machines without a GPU: a call that is not refused would run on made-up pointers")
    lib, ctx = moe.load_library(), ctypes.create_string_buffer(b"\x40" * 4096, 4096)

    def status(grads, outs, counts, types):
        n = len(grads)
        put = lambda places: (ctypes.c_void_p * n)(*[p if p is None else BASE + p for p in places])  # noqa: E731
        return lib.moe_clip_grads(ctypes.addressof(ctx), put(grads), (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*types), n, BASE - 64, 1.0,
                                  None if outs is None else put(outs))
    return status


BF16, F32 = 0, 1


def test_places(clip):
    two, f32 = [10, 10], [F32, F32]
    assert clip([0, 40], [40, 0], two, f32) == REFUSED                     # changed about
    assert clip([0, 40], [80, 0], two, f32) == REFUSED                     # over the one, in front of its own
    assert clip([0, 40], [76, 200], two, f32) == REFUSED                   # over an end
    assert clip([0, 40], [200, 36], two, f32) == REFUSED                   # over the other's end, and its own place
    assert clip([0, 40], [0, 0], two, f32) == REFUSED                      # in place, and over it
    assert clip([40, 0], [0, 40], [10, 0], f32) == PASSED_ON               # (nothing is there to be overwritten)
    assert clip([None, 0], [None, 40], [0, 10], f32) == PASSED_ON
    for outs in ([80, 120], [0, 40], [0, 80], [80, 40], None):
        assert clip([0, 40], outs, two, f32) == PASSED_ON, outs
    assert clip([0, 80], [40, 120], two, f32) == PASSED_ON                 # one of each in turn
    assert clip([0, 60], [20, 40], two, [BF16, BF16]) == PASSED_ON
    assert clip([0, 60], [20, 42], two, [BF16, BF16]) == REFUSED


def test_lists_in_any_order(clip):
    """Against every pair of an output and another's gradient, or its own at another place."""
    rng = random.Random(7)
    seen = {REFUSED: 0, PASSED_ON: 0}
    for _ in range(600):
        n = rng.choice([1, 2, 3, 5, 40, 128])
        counts, types = [rng.choice([0, 1, 3, 50]) for _ in range(n)], [rng.choice([F32, BF16]) for _ in range(n)]
        sizes = [c * (2 if t == BF16 else 4) for c, t in zip(counts, types)]
        places, at = [], 0
        for k in rng.sample(range(2 * n), 2 * n):
            places.append((k, at))
            at += -(-sizes[k % n] // 4) * 4 + rng.choice([0, 0, 4])
        place = dict(places)
        grads = [place[k] for k in range(n)]
        outs = [grads[k] if rng.random() < 0.3 else place[n + k] for k in range(n)]
        if rng.random() < 0.6:
            k = rng.randrange(n)
            outs[k] = max(0, rng.choice(grads + outs) + rng.choice([-4, 0, 4]))
        if rng.random() < 0.2:
            order = sorted(range(n), key=lambda k: grads[k])
            grads, outs, counts, types, sizes = ([v[k] for k in order] for v in (grads, outs, counts, types, sizes))
        some = [k for k in range(n) if sizes[k]]
        bad = any(outs[j] < grads[k] + sizes[k] and grads[k] < outs[j] + sizes[j] and (j, outs[j]) != (k, grads[k]) for j in some for k in some)
        got = clip(grads, outs, counts, types)
        if sum(counts) == 0:
            assert got == 0
            continue
        assert got == (REFUSED if bad else PASSED_ON), (grads, outs, counts, types)
        seen[got] += 1
    assert min(seen.values()) > 100, seen
