"""The 8-bit K/V cache where it is easily got wrong: sequences that sit a call out, blocks whose scales lie far apart, waits that run
out, sizes at the ends of their ranges. References in kv8_ref; the bounds stand beside the tests."""
import numpy as np
import pytest
import torch

from . import kv8_ref as R
from .test_gpu_kv8 import _bd, _bf16, _cache, _same_cache, _shape, _to_gpu

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("idle", [0, -3])
def test_append_does_not_touch_a_sequence_that_sits_out(idle):
    """Slots that a server has freed or paused, each with a length inside a block: no table entry, a length beyond every slot, scales
    that no append writes (too small, zero, NaN). Nothing is flagged, no byte changes but the one active sequence's."""
    Bd, rng = _bd(), np.random.default_rng(61)
    Hkv, dh, page, M = 2, 64, 16, 3
    ctx = Bd.Context(_shape(4, Hkv, dh, page), max_rows=64, max_K=1, max_ctx=512)
    lens = [5, 21, 9, 3, 7, 12]
    kv = _cache(rng, Hkv, dh, page, lens, M)
    first = kv["block_table"][:, 0].copy()
    kv["block_table"][0] = -1
    kv["seq_lens"][1] = 200                               # there are slots for 32
    for b, s in ((2, 2.0 ** -130), (3, 0.0), (4, np.nan)):
        for w in "kv":
            kv[w + "_scales"][first[b]] = s
    n_new = [idle] * 5 + [M]
    dev = _to_gpu(kv)
    x, ref = _bf16(rng, (6, M, Hkv, dh))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_kv8_append(x, x, Bd.kv8(dev), 6, M, n_new=_i32(n_new), dev_status=st)
    for w in "kv":
        R.append(kv, w, ref, [max(0, n) for n in n_new], page)
    _same_cache(dev, kv)
    assert int(st.item()) == 0
    ctx.close()


def test_append_beside_an_idle_holder_of_the_same_block():
    """An idle sequence's last block has been given to one that appends in the same call, and two calls on two streams take turns over
    one cache with complementary rows: what is written is the active side's, whose scales grow all the time."""
    Bd, rng = _bd(), np.random.default_rng(62)
    Hkv, dh, page, M, half = 4, 128, 16, 2, 24
    shape = _shape(8, Hkv, dh, page)
    ctxs = [Bd.Context(shape, max_rows=8, max_K=1, max_ctx=512) for _ in range(2)]
    lens = [1 + int(v) for v in rng.integers(0, 14, 2 * half)]
    kv = _cache(rng, Hkv, dh, page, lens, 4 * M + page)
    for b in range(0, 2 * half, 4):                       # b sits out in the calls that append to b + 1
        kv["block_table"][b] = kv["block_table"][b + 1]
        lens[b] = lens[b + 1]
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    sides = [[M if b % 4 == 1 else 0 for b in range(2 * half)], [M if b % 4 in (2, 3) else 0 for b in range(2 * half)]]
    dev = _to_gpu(kv)
    streams = [torch.cuda.Stream() for _ in ctxs]
    counts = [_i32(s) for s in sides]
    for step in range(4):
        rows = [_bf16(rng, (2 * half, M, Hkv, dh), 4.0 ** step) for _ in ctxs]
        torch.cuda.synchronize()
        for c, s, n, (x, _) in zip(ctxs, streams, counts, rows):
            c.fastmtp_kv8_append(x, x, Bd.kv8(dev), 2 * half, M, n_new=n, stream=s)
        torch.cuda.synchronize()
        for n, (_, ref) in zip(sides, rows):
            for w in "kv":
                R.append(kv, w, ref, n, page)
        _same_cache(dev, kv)
        moved = np.asarray([sides[0][b] + sides[1][b] for b in range(2 * half)], dtype=np.int32)
        moved[0::4] = moved[1::4]
        kv["seq_lens"] = kv["seq_lens"] + moved
        dev["seq_lens"] += torch.from_numpy(moved).cuda()
    for c in ctxs:
        c.close()
