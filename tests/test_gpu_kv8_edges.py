"""The 8-bit K/V cache where it is easily got wrong: sequences that sit a call out, blocks whose scales lie far apart, waits that run
out, sizes at the ends of their ranges. References in kv8_ref; the bounds stand beside the tests."""
import time

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


def _attention(kv, q, n_new, page):
    """q [B, M, Hq, dh] float64 -> (out, bound), NaN and 0 in rows that do not count. The bound, element by element, from what the
    header says of the kernels:

    * the output is bf16: 2^-8 of it;
    * a weight, w_t = (probability of token t) * (its V scale), is rounded to f16: 2^-11 of itself, or 2^-27 of the row's and head's
      largest weight (never more than the weight itself, which then counts as nothing), times the token's code;
    * a score is off by 2^-20 of the sum of its products' magnitudes (products of codes and query elements are exact, fp32 adds
      them, an MMA keeps 22 bits of the largest), and in tiles of 128 pairs by what a query element below 2^-9 of the row's largest loses
      in two e4m3 parts, half of a smallest step (2^-10 where the largest lies in 224 .. 448): twice the largest such error
      enters the output, once above and once below the fraction;
    * 2^-14 for the powers of two, the scales' logarithms (2^-22 of up to 120) and fp32 sums and joins."""
    B, M, Hq, dh = q.shape
    hkv = kv["k_pages"].shape[1]
    g = Hq // hkv
    tiles = M * g > 32 and dh == 128 and page % 16 == 0
    ones = {**kv, "v_scales": np.ones_like(kv["v_scales"])}
    out, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    for b in range(B):
        if not n_new[b]:
            continue
        L = int(kv["seq_lens"][b])
        T = min(L + int(n_new[b]), kv["block_table"].shape[1] * page)
        K, V, code = R.tokens(kv, "k", b, T, page), R.tokens(kv, "v", b, T, page), np.abs(R.tokens(ones, "v", b, T, page))
        pg = kv["block_table"][b, np.arange(T) // page]
        S = kv["v_scales"][pg].astype(np.float64)
        for m in range(int(n_new[b])):
            n = min(L + m + 1, T)
            for h in range(Hq):
                k, v, qv = K[:n, h // g], V[:n, h // g], q[b, m, h]
                s = k @ qv / np.sqrt(dh)
                p = np.exp(s - s.max())
                p /= p.sum()
                o, mass = p @ v, p @ np.abs(v)
                serr = 2.0 ** -20 * (np.abs(k) @ np.abs(qv)).max()
                if tiles:
                    big = np.abs(qv).max()
                    serr += big * 2.0 ** -10 / 224 * (np.abs(k) @ (np.abs(qv) < 2.0 ** -9 * big)).max()
                w = p * S[:n, h // g]
                small = np.minimum(w, 2.0 ** -27 * w.max()) @ code[:n, h // g]
                out[b, m, h] = o
                tol[b, m, h] = 2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2.0 ** -14 + 2 * serr / np.sqrt(dh)) * mass + 1.01 * small
    return out, tol


def _attend(Bd, ctx, dev, q, n_new=None):
    B, M = q.shape[:2]
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, out, n_new=None if n_new is None else _i32(n_new), dev_status=st)
    assert int(st.item()) == 0
    return out


def _within(got, ref, tol, what=""):
    err = np.abs(got.double().cpu().numpy() - ref)
    assert np.all(err <= tol), (what, float((err / tol).max()), np.argwhere(~(err <= tol))[:3])


# one and two tiles of eight pairs per set, two tiles per warp (64-wide heads; blocks of 5), tiles of 128 pairs
FORMS = [(8, 1, 128, 16, 1), (28, 4, 128, 16, 4), (8, 2, 64, 16, 1), (8, 1, 64, 16, 3), (8, 1, 64, 16, 8), (8, 1, 128, 5, 6), (8, 1, 128, 16, 8),
         (28, 4, 128, 16, 64)]


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", FORMS)
@pytest.mark.parametrize("apart", [5, 18, 36, 100])
def test_attention_where_scales_lie_far_apart(Hq, Hkv, dh, page, M, apart):
    """A few blocks hold nearly all of the probability and have V scales 2^-apart of the others', whose products with their probabilities
    are less still; for some heads it is the other way round. One block's scale is zero."""
    Bd, rng = _bd(), np.random.default_rng(71 + apart)
    lens = [700, 150, 40]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=3 * M, max_K=1, max_ctx=1024)
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M, garbage=False)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    far = (apart * np.log(2.0) + 9) / np.sqrt(dh)         # a key of that size everywhere: a score 9 and more below what the scales lie apart
    for b, L in enumerate(lens):
        blocks = -(-(L + M) // page)
        heavy = {0: (0,), 1: (blocks // 2,), 2: (blocks - 1,)}[b] + (blocks // 3,)
        for i in range(blocks):
            pg, low = kv["block_table"][b, i], i in heavy
            kv["k_scales"][pg] = R.scale_for(far)
            kv["k_pages"][pg] = R.encode(np.where(low, 0.0, -far / R.scale_for(far)) + 2.0 ** -9 * rng.integers(-2, 3, kv["k_pages"][pg].shape))
            kv["v_scales"][pg] = 2.0 ** ((0 if low else apart) - 8 + int(rng.integers(0, 3)))
        kv["v_scales"][kv["block_table"][b, blocks // 2 - 1]] = 0.0
    qr = np.ones((3, M, Hq, dh))
    qr[:, :, 1::4] = -0.25
    q = torch.from_numpy(qr.astype(np.float32)).to(torch.bfloat16).cuda()
    out = _attend(Bd, ctx, _to_gpu(kv), q)
    _within(out, *_attention(kv, qr, [M] * 3, page))
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", [f for f in FORMS if f[4] > 1])
def test_attention_rows_do_not_meet_later_rows_scales(Hq, Hkv, dh, page, M):
    """A later row opens a block whose scales are enormous (its values are): the rows before it give the bits they give without it."""
    Bd, rng = _bd(), np.random.default_rng(81)
    back = min(M - 1, 2)                                  # rows before the new block
    lens = [page - back, 20 * page - back, 5 * page - 1]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=3 * M, max_K=1, max_ctx=1024)
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M, garbage=False)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, qr = _bf16(rng, (3, M, Hq, dh), 1.5)
    good = _attend(Bd, ctx, dev, q)
    _within(good, *_attention(kv, qr, [M] * 3, page))
    for b, L in enumerate(lens):
        for blk in range(-(-L // page), -(-(L + M) // page)):
            for w in "kv":
                kv[w + "_scales"][kv["block_table"][b, blk]] *= np.float32(2.0 ** (50 if w == "v" else 3))
    out = _attend(Bd, ctx, _to_gpu(kv), q)
    for b, L in enumerate(lens):
        n = -(-L // page) * page - L
        assert n > 0 and torch.equal(good[b, :n], out[b, :n]), b
    _within(out, *_attention(kv, qr, [M] * 3, page))
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,M,B", [(8, 1, 8, 3), (28, 4, 64, 2)])
def test_a_wait_of_the_tiles_of_pairs_that_runs_out_leaves_the_context_usable(Hq, Hkv, M, B):
    """The next call's stages of keys expect one copy more than is made and its waits are limited to 20 ms: it returns soon after with
    the timeout flag, and the same call then gives the bits it gave before. An armed context's smaller calls do not wait."""
    Bd, rng = _bd(), np.random.default_rng(91)
    dh, page = 128, 16
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=B * M, max_K=1, max_ctx=2048)
    lens = [900, 1500, 30][:B]
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M, garbage=False)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, qr = _bf16(rng, (B, M, Hq, dh))
    want = _attend(Bd, ctx, dev, q)
    _within(want, *_attention(kv, qr, [M] * B, page))
    for _ in range(2):
        out, st = torch.zeros_like(want), torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        ctx.fmtp_selftest_inject_wait_timeout(20, 4)
        t0 = time.time()
        ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, out, dev_status=st)
        torch.cuda.synchronize()
        assert int(st.item()) == Bd.DEV_TIMEOUT and 0.015 < time.time() - t0 < 2.0
        assert torch.equal(_attend(Bd, ctx, dev, q), want)
    ctx.fmtp_selftest_inject_wait_timeout(20, 4)
    _attend(Bd, ctx, dev, q[:, :1].contiguous())          # (eight pairs: no tiles, and the arming is used up)
    assert torch.equal(_attend(Bd, ctx, dev, q), want)
    with pytest.raises(Bd.FastMTPError):
        ctx.fmtp_selftest_inject_wait_timeout(20, 5)
    ctx.close()


def test_read_of_nothing_from_beyond_every_slot():
    """A start beyond every slot is no fault where nothing is asked for from there."""
    Bd, rng = _bd(), np.random.default_rng(101)
    Hkv, dh, page = 2, 64, 16
    ctx = Bd.Context(_shape(4, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=4096)
    kv = _cache(rng, Hkv, dh, page, [20, 60, 33], 0)
    dev = _to_gpu(kv)
    out = [torch.full((3, 64, Hkv, dh), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_kv8_read(Bd.kv8(dev), 3, 64, *out, start=_i32([64, 5000, 2 ** 31 - 1]), count=_i32([0, -1, 0]), dev_status=st)
    ctx.fastmtp_kv8_read(Bd.kv8(dev), 3, 64, *out, start=_i32([64, 5000, 2 ** 31 - 1]), dev_status=st)       # all that is committed from there on
    assert int(st.item()) == 0 and all(bool((o == 7.0).all()) for o in out)
    ctx.fastmtp_kv8_read(Bd.kv8(dev), 3, 64, *out, start=_i32([64, 0, 0]), count=_i32([1, 0, 0]), dev_status=st)
    assert int(st.item()) == Bd.DEV_BAD_POS and all(bool((o == 7.0).all()) for o in out)
    ctx.close()


def test_read_into_room_for_more_than_there_is():
    """max_n is the caller's stride; only what there is to read takes part, whatever its size."""
    Bd, rng = _bd(), np.random.default_rng(102)
    Hkv, dh, page = 2, 64, 16
    ctx = Bd.Context(_shape(4, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=4096)
    kv = _cache(rng, Hkv, dh, page, [60], 0)
    dev = _to_gpu(kv)
    for max_n in (1000, 2 ** 31 - 1):
        out = [torch.full((64, Hkv, dh), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.fastmtp_kv8_read(Bd.kv8(dev), 1, max_n, *out, dev_status=st)
        for w, o in zip("kv", out):
            assert np.array_equal(o[:60].double().cpu().numpy(), R.tokens(kv, w, 0, 60, page)) and bool((o[60:] == 7.0).all())
        assert int(st.item()) == 0
    ctx.close()


def test_append_takes_as_many_rows_as_a_sequence_may_have_positions():
    Bd, rng = _bd(), np.random.default_rng(103)
    Hkv, dh, page = 2, 64, 16
    ctx = Bd.Context(_shape(4, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=100)
    kv = _cache(rng, Hkv, dh, page, [0], 112)
    dev = _to_gpu(kv)
    x, ref = _bf16(rng, (1, 101, Hkv, dh))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_kv8_append(x, x, Bd.kv8(dev), 1, 100, dev_status=st)
    for w in "kv":
        R.append(kv, w, ref, [100], page)
    _same_cache(dev, kv)
    assert int(st.item()) == 0
    with pytest.raises(Bd.FastMTPError) as e:
        ctx.fastmtp_kv8_append(x, x, Bd.kv8(dev), 1, 101)
    assert e.value.code == -2
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", FORMS + [(4, 2, 64, 16, 64), (16, 16, 64, 32, 3), (5, 5, 64, 24, 33), (6, 3, 128, 1, 3), (64, 8, 128, 64, 1),
                                                      (64, 8, 128, 48, 16), (28, 4, 128, 32, 19), (32, 8, 128, 64, 4)])
def test_attention_is_as_near_as_the_header_says_and_repeats_itself(Hq, Hkv, dh, page, M):
    """Random values in caches as they are filled, scores from even to peaked, lengths at the edges of stages, blocks and chunks, rows
    that do not count, single-token contexts; four calls give the same bits."""
    Bd, rng = _bd(), np.random.default_rng(Hq * 11 + M * 5 + page)
    lens = [0, 1, 31, 32, 127, 129, 511, 40, 1100] if M <= 8 else [0, 31, 127, 40, 600]
    B = len(lens)
    n_new = [M] * (B - 2) + [max(1, M // 2), M]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=B * M, max_K=1, max_ctx=2048)
    kv = _cache(rng, Hkv, dh, page, [L + n for L, n in zip(lens, n_new)], M)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, _ = _bf16(rng, (B, M, Hq, dh))
    q *= (2.0 ** torch.from_numpy(rng.integers(-6, 3, (B, M, Hq, 1))).double()).to(torch.bfloat16).cuda()
    out = _attend(Bd, ctx, dev, q, n_new)
    ref, tol = _attention(kv, q.double().cpu().numpy(), n_new, page)
    for b, n in enumerate(n_new):
        _within(out[b, :n], ref[b, :n], tol[b, :n], b)
    for _ in range(3):
        assert torch.equal(_attend(Bd, ctx, dev, q, n_new), out)
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page,M,B", [(28, 4, 128, 16, 1, 64), (28, 4, 128, 16, 4, 17), (28, 4, 128, 16, 64, 4), (32, 8, 128, 16, 1, 2),
                                                (16, 2, 64, 16, 6, 40), (16, 2, 64, 5, 1, 64)])
def test_attention_of_full_batches_repeats_itself(Hq, Hkv, dh, page, M, B):
    """All SMs busy with ragged contexts, four calls in a row beside a copy on another stream, ten times over: the same bits each time."""
    Bd, rng = _bd(), np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 30000 if B == 2 else 5000, B)]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=B * M, max_K=1, max_ctx=32768)
    per = [-(-(L + M) // page) for L in lens]
    g = torch.Generator(device="cuda").manual_seed(B)
    num = sum(per) + 1
    order = torch.randperm(num, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, max(per)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, p in enumerate(per):
        table[b, :p] = order[at:at + p]
        at += p
    dev = {"block_table": table, "seq_lens": _i32(lens)}
    for w in "kv":
        x = torch.randn((num, Hkv, page, dh), generator=g, device="cuda")
        dev[w + "_pages"] = (x * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        dev[w + "_scales"] = 2.0 ** torch.randint(-9, -4, (num, Hkv), generator=g, device="cuda").float()
    q = torch.randn((B, M, Hq, dh), generator=g, device="cuda").to(torch.bfloat16)
    want = _attend(Bd, ctx, dev, q)
    assert bool(torch.isfinite(want.float()).all())
    side, big = torch.cuda.Stream(), torch.zeros(1 << 27, device="cuda")
    outs = [torch.zeros_like(want) for _ in range(4)]
    for _ in range(10):
        with torch.cuda.stream(side):
            big.add_(1.0)
        for o in outs:
            o.zero_()
            ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, o)
        assert all(torch.equal(o, want) for o in outs)
    ctx.close()


def test_speculative_decoding_over_8_bit_caches_stays_with_greedy():
    """Rejected drafts may raise a block's scale, and rows scored together are cut into other chunks: the two are not the same bits. They
    emit the same tokens up to a near tie (the bound of gpu_util and one bf16 spacing of the logit, as for the target step's own
    greedy token), behind which they go separate ways."""
    from paper_2509_18362_b200 import inputs as I
    from paper_2509_18362_b200 import loop

    from .gpu_util import GAP_TOL
    Bd, shape, K, n_new, room = _bd(), I.TINY.with_layers(2), 3, 48, 128
    for seed in (701, 702):
        Wt = I.target_weights(shape, seed)
        Wm = I.mtp_weights(shape, seed + 1, embed=Wt["embed"], lm_head=Wt["lm_head"])
        prompt = [int(t) for t in I.token_ids(seed + 2, (21,), shape.vocab)]
        ids = torch.from_numpy(I.subset_uniform(shape.vocab, 1024, seed + 3)).cuda()
        ctx = Bd.Context(shape, max_rows=64, max_K=8, max_ctx=room)
        dW = Bd.to_device(Wt)
        blocks = room // shape.page_size
        pool = (blocks + 1, shape.n_kv_heads, shape.page_size, shape.head_dim)

        def target():
            return loop.Target(ctx, shape, dW, [dict({w + "_pages": torch.zeros(pool, dtype=torch.uint8, device="cuda") for w in "kv"},
                                                     **{w + "_scales": torch.ones(pool[:2], device="cuda") for w in "kv"},
                                                     block_table=_i32([np.random.default_rng(seed + l).permutation(blocks + 1)[:blocks].tolist()]),
                                                     seq_lens=_i32([0])) for l in range(shape.n_layers)])

        plain = target()
        _, tok = loop.prefill(plain, prompt)
        ref, gaps = [tok], [0.0]
        while len(ref) < n_new + K + 1:
            _, logits, a = plain.step([[ref[-1]]], want_logits=True)
            plain.advance(1)
            top = torch.topk(logits[0, 0].double(), 2).values.tolist()
            gaps.append((top[0] - top[1]) - 2.0 ** -7 * abs(top[0]))       # (a bf16 spacing is 2^-7 of the value at most)
            ref.append(int(a.item()))

        def inject(rnd, K, emitted):
            good = ref[emitted:emitted + K]
            n_ok = rnd % (K + 1)
            return list(good[:n_ok]) + [(t + 1) % shape.vocab for t in good[n_ok:]]

        dWm = dict(Bd.to_device({k: v for k, v in Wm.items() if k not in ("embed", "lm_head")}), embed=dW["embed"], lm_head=dW["lm_head"])
        mkv = Bd.to_device(I.empty_paged_kv(shape, 1, room, seed + 20))
        tgt = target()
        out, stats = loop.speculative_decode(tgt, Bd.mtp_w(dWm), mkv, ids, prompt, n_new, K, inject)
        apart = next((i for i in range(n_new) if out[i] != ref[i]), n_new)
        assert apart > 0 and (apart == n_new or gaps[apart] < GAP_TOL), (apart, gaps[apart])
        print(f"8-bit caches, seed {seed}: {apart} of {n_new} tokens alike, accepted {stats['accepted']}")
        assert apart < n_new or {0, 1, 2, 3} <= set(stats["accepted"])
        ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", FORMS)
@pytest.mark.parametrize("low,high,span", [(112, 115, 0), (110, 117, 5), (-132, -127, 0), (-134, -120, 5)])
def test_attention_over_values_near_the_ends_of_the_numbers(Hq, Hkv, dh, page, M, low, high, span):
    """Scales of blocks between 2^low and 2^high (and single ones 2^span beyond): values up to 2^126 whose mean is a finite number, and
    values below 2^-111 under scales that have lost bits themselves. (Beside the bound, half a step of the smallest bf16, 2^-134,
    and of fp32's, 2^-150, of each of 32 sums.)"""
    Bd, rng = _bd(), np.random.default_rng(111 + M)
    lens = [700, 33, 5]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=3 * M, max_K=1, max_ctx=1024)
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M, garbage=False)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    kv["v_scales"][:] = 2.0 ** rng.integers(low, high + 1, kv["v_scales"].shape)
    if span:
        kv["v_scales"][rng.random(kv["v_scales"].shape) < 0.2] = 2.0 ** (high + span if high > 0 else low - span)
    if high > 0:                                          # codes below 16: values below 2^126
        kv["v_pages"] = R.encode(R.TABLE[kv["v_pages"]] / 32)
    q, qr = _bf16(rng, (3, M, Hq, dh))
    out = _attend(Bd, ctx, _to_gpu(kv), q)
    ref, tol = _attention(kv, qr, [M] * 3, page)
    _within(out, ref, tol + 2.0 ** -134 + 32 * 2.0 ** -150)
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", FORMS)
@pytest.mark.parametrize("keys", [105, 60, -60, -105])
def test_attention_of_large_keys_and_small_queries(Hq, Hkv, dh, page, M, keys):
    """Keys times 2^keys under queries times 2^-keys: the scores are those of neither."""
    Bd, rng = _bd(), np.random.default_rng(121 + M)
    lens = [300, 33, 5]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=3 * M, max_K=1, max_ctx=1024)
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M, garbage=False)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    kv["k_scales"] = (kv["k_scales"].astype(np.float64) * 2.0 ** keys).astype(np.float32)
    q, _ = _bf16(rng, (3, M, Hq, dh))
    q = (q.double() * 2.0 ** -keys).to(torch.bfloat16)
    out = _attend(Bd, ctx, _to_gpu(kv), q)
    _within(out, *_attention(kv, q.double().cpu().numpy(), [M] * 3, page))
    ctx.close()
