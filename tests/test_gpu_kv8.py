"""The 8-bit K/V cache on the GPU: quantising into it (exact), reading back (exact), attention over it (bounds derived in
kv8_ref.attention) and the target step that uses both."""
import numpy as np
import pytest
import torch

from oracle import fastmtp_oracle as O
from paper_2509_18362_b200 import inputs as I

from . import kv8_ref as R
from .gpu_util import close, copy_kv

pytestmark = pytest.mark.gpu


def _bd():
    from paper_2509_18362_b200 import binding as Bd
    return Bd


def _shape(Hq, Hkv, dh, page):
    return I.Shape(d=128, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=dh, ffn=64, vocab=64, n_layers=1, page_size=page)


def _cache(rng, Hkv, dh, page, lens, room, garbage=True, spare=3):
    """Numpy cache of the given committed lengths: random codes and scales where something is committed, NaN elsewhere."""
    B = len(lens)
    per = [max(1, -(-(int(L) + room) // page)) for L in lens]
    num = sum(per) + spare
    perm = rng.permutation(num).astype(np.int32)
    table = np.full((B, max(per)), -1, dtype=np.int32)
    at = 0
    for b, p in enumerate(per):
        table[b, :p] = perm[at:at + p]
        at += p
    kv = {"block_table": table, "seq_lens": np.asarray(lens, dtype=np.int32)}
    for w in "kv":
        x = rng.standard_normal((num, Hkv, page, dh)) * 2.0 ** rng.standard_normal((1, Hkv, 1, dh))
        s = np.array([R.scale_for(a) for a in np.abs(x).max(axis=(2, 3)).ravel()]).reshape(num, Hkv)
        codes = R.encode(x / s[:, :, None, None])
        if garbage:
            used = np.zeros((num, page), bool)
            for b, L in enumerate(lens):
                for blk in range(-(-int(L) // page)):
                    used[table[b, blk], :min(page, int(L) - blk * page)] = True
            codes[~used[:, None, :].repeat(Hkv, 1)] = R.NAN_CODE
            s[~used.any(axis=1)] = np.nan
        kv[w + "_pages"], kv[w + "_scales"] = codes, s.astype(np.float32)
    return kv


def _to_gpu(kv):
    return {k: torch.from_numpy(np.ascontiguousarray(v)).cuda() for k, v in kv.items()}


def _bf16(rng, shape, std=1.0):
    x = torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(torch.bfloat16)
    return x.cuda(), x.double().numpy()


def _same_cache(dev, kv):
    for k in ("k_pages", "v_pages"):
        got = dev[k].cpu().numpy()
        bad = np.argwhere(got != kv[k])
        assert bad.size == 0, (k, bad[:4], got[tuple(bad[0])], kv[k][tuple(bad[0])])
    for k in ("k_scales", "v_scales"):
        assert np.array_equal(dev[k].cpu().numpy(), kv[k], equal_nan=True), k


LAYOUTS = [(28, 4, 128, 16), (4, 2, 64, 16), (16, 16, 64, 32), (8, 1, 128, 5), (6, 3, 128, 1), (64, 8, 128, 64), (5, 5, 64, 24)]


@pytest.mark.parametrize("Hq,Hkv,dh,page", LAYOUTS)
def test_append_gives_the_bytes_of_the_definition(Hq, Hkv, dh, page):
    """Codes and scales, committed codes of partly filled blocks among them; the rest of the pool is left alone; a second call on the
    same inputs changes nothing."""
    Bd, rng = _bd(), np.random.default_rng(Hq * 1000 + page)
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=4096)
    for M in (1, 3, page, 2 * page + 3, 70):
        lens = [0, 1, page - 1, page, page + 1, 3 * page + page // 2, 100]
        n_new = [M, M, 0, max(1, M - 1), M, M // 2, M]
        kv = _cache(rng, Hkv, dh, page, lens, M + 2)
        dev = _to_gpu(kv)
        wide = (Hq + 2 * Hkv) * dh
        rows, ref = _bf16(rng, (len(lens) * M, wide), 4.0)
        rows[::3] *= 64                                   # blocks whose scale has to grow, and some that stay
        ref = rows.double().cpu().numpy().reshape(len(lens), M, Hq + 2 * Hkv, dh)
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        for _ in range(2):
            ctx.fastmtp_kv8_append(rows[:, Hq * dh:], rows[:, (Hq + Hkv) * dh:], Bd.kv8(dev), len(lens), M,
                                   n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"), dev_status=st, ld=wide)
        R.append(kv, "k", ref[:, :, Hq:Hq + Hkv], n_new, page)
        R.append(kv, "v", ref[:, :, Hq + Hkv:], n_new, page)
        _same_cache(dev, kv)
        assert int(st.item()) == 0
    ctx.close()


def test_append_extremes_and_growth_token_by_token():
    """Infinities, NaN, zeros, the smallest and largest numbers; scales that grow while a block fills."""
    Bd, rng = _bd(), np.random.default_rng(5)
    Hkv, dh, page = 2, 64, 16
    ctx = Bd.Context(_shape(4, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=512)
    kv = _cache(rng, Hkv, dh, page, [0, 7], 40)
    dev = _to_gpu(kv)
    for step in range(36):
        x = rng.standard_normal((2, 1, Hkv, dh)) * 2.0 ** (step % 7 * 3 - 9)
        if step == 3:
            x[0] = 0.0
        if step == 5:
            x[0, 0, 0, :4] = [np.inf, -np.inf, np.nan, 1.0]
        if step == 9:
            x[1] = np.nan
        if step == 17:
            x[0, 0, 1, :3] = [2.0 ** -133, -2.0 ** -126, 1e-39]
            x[0, 0, 1, 3:] = 0
        if step == 33:
            x[1, 0, 1, 0] = -1.5 * 2.0 ** 126
        xb = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16)
        ctx.fastmtp_kv8_append(xb.cuda(), (2 * xb).cuda(), Bd.kv8(dev), 2, 1)
        R.append(kv, "k", xb.double().numpy(), [1, 1], page)
        R.append(kv, "v", (2 * xb).double().numpy(), [1, 1], page)
        kv["seq_lens"] = kv["seq_lens"] + 1
        dev["seq_lens"] += 1
        _same_cache(dev, kv)
    ctx.close()


def test_append_skips_positions_without_a_slot_and_bad_pages():
    Bd, rng = _bd(), np.random.default_rng(6)
    Hkv, dh, page = 2, 64, 16
    ctx = Bd.Context(_shape(4, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=512)
    kv = _cache(rng, Hkv, dh, page, [30, 5, 20], 2)
    cap = kv["block_table"].shape[1] * page               # 32
    kv["block_table"][1, 0] = kv["k_pages"].shape[0]      # out of range
    kv["block_table"][2, 1] = -7
    dev = _to_gpu(kv)
    x, ref = _bf16(rng, (3, 4, Hkv, dh))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_kv8_append(x, x, Bd.kv8(dev), 3, 4, dev_status=st)
    R.append(kv, "k", ref, [4, 4, 4], page)
    R.append(kv, "v", ref, [4, 4, 4], page)
    _same_cache(dev, kv)
    assert cap == 32 and int(st.item()) == Bd.DEV_BAD_POS | Bd.DEV_BAD_PAGE
    dev["seq_lens"][:] = torch.tensor([2 ** 31 - 1, -5, 2 ** 30 + 7], dtype=torch.int32)      # no such lengths: nothing is written but at 0
    before = dev["k_pages"].clone()
    ctx.fastmtp_kv8_append(x[:1], x[:1], Bd.kv8({**dev, "seq_lens": dev["seq_lens"][:1]}), 1, 4, dev_status=st)
    ctx.fastmtp_kv8_append(x[2:], x[2:], Bd.kv8({**dev, "seq_lens": dev["seq_lens"][2:]}), 1, 4, dev_status=st)
    assert torch.equal(before, dev["k_pages"])
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page", LAYOUTS)
def test_read_gives_the_values(Hq, Hkv, dh, page):
    Bd, rng = _bd(), np.random.default_rng(Hq + page)
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=4096)
    lens = [0, 1, 16, 133, 64]
    kv = _cache(rng, Hkv, dh, page, lens, 4)
    dev = _to_gpu(kv)
    for start, count, max_n in ((None, None, 133), (None, None, 40), ([0, 1, 15, 60, 3], [0, 0, 1, 50, 61], 55), ([5, 0, 3, 130, 64], None, 20)):
        s = start or [0] * 5
        n = [min(max_n, c) for c in (count or [max(0, L - a) for L, a in zip(lens, s)])]
        n = [min(x, max(0, dev["block_table"].shape[1] * page - a)) for x, a in zip(n, s)]
        out = [torch.full((5, max_n, Hkv, dh), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        i32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        ctx.fastmtp_kv8_read(Bd.kv8(dev), 5, max_n, out[0], out[1], start=i32(start), count=i32(count))
        for w, o in zip("kv", out):
            want = np.full(o.shape, 7.0)
            for b in range(5):
                if n[b]:
                    want[b, :n[b]] = R.tokens(kv, w, b, s[b] + n[b], page)[s[b]:]
            assert np.array_equal(o.double().cpu().numpy(), want, equal_nan=True), (w, start, max_n)      # four bits: exact in bf16
    ctx.close()


def _attend(Bd, ctx, dev, q, B, M, n_new, out=None, **kw):
    Hq, dh = q.shape[-2:]
    out = torch.full((B, M, Hq, dh), 9.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    nn = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, out, n_new=nn, dev_status=st, **kw)
    return out, st


def _committed(kv, n_new):
    """The cache as it stands after the rows were appended: garbage starts behind them."""
    return [int(L) + int(n) for L, n in zip(kv["seq_lens"], n_new)]


CASES = [  # Hq, Hkv, dh, page, M: every kernel variant (8, 16, 32, 64 pairs, several sets), both head dimensions
    (28, 4, 128, 16, 1), (28, 4, 128, 16, 2), (28, 4, 128, 16, 4), (28, 4, 128, 16, 7), (28, 4, 128, 16, 19),
    (4, 2, 64, 16, 1), (4, 2, 64, 16, 5), (4, 2, 64, 16, 64), (16, 16, 64, 32, 1), (16, 16, 64, 32, 3), (5, 5, 64, 24, 33),
    (8, 1, 128, 5, 1), (8, 1, 128, 5, 2), (6, 3, 128, 1, 3), (64, 8, 128, 64, 1), (64, 8, 128, 64, 8), (32, 8, 128, 64, 4),
]


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", CASES)
def test_attention_against_64_bits(Hq, Hkv, dh, page, M):
    """Lengths from nothing committed to several chunks, rows that sit out, garbage (NaN) in every slot that nothing was written to."""
    Bd, rng = _bd(), np.random.default_rng(Hq * 7 + M * 13 + page)
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=24 * M, max_K=1, max_ctx=4096)
    lens = [0, 1, 2, 15, 16, 17, 30, 31, 32, 33, 63, 64, 127, 128, 129, 255, 256, 257, 511, 513, 1300, 40, 0, 77]
    if M > 8:
        lens = [0, 1, 31, 33, 250, 700, 40, 77]
    B = len(lens)
    n_new = [M] * (B - 3) + [0, max(1, M // 2), max(1, M - 1)]
    kv = _cache(rng, Hkv, dh, page, [L + n for L, n in zip(lens, n_new)], M)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, qr = _bf16(rng, (B, M, Hq, dh), 1.5)
    out, st = _attend(Bd, ctx, dev, q, B, M, n_new)
    ref, tol = R.attention(kv, qr, n_new, page)
    got = out.double().cpu().numpy()
    for b in range(B):
        assert np.all(got[b, n_new[b]:] == 9.0), b        # rows that do not count
        if n_new[b]:
            err = np.abs(got[b, :n_new[b]] - ref[b, :n_new[b]])
            assert np.all(np.isfinite(err)), (b, lens[b])
            assert np.all(err <= tol[b, :n_new[b]]), (b, lens[b], float((err / tol[b, :n_new[b]]).max()))
    assert int(st.item()) == 0
    # a sequence alone: the same bits as in the batch
    b = B - 4
    one = {**dev, "block_table": dev["block_table"][b:b + 1].contiguous(), "seq_lens": dev["seq_lens"][b:b + 1]}
    alone, _ = _attend(Bd, ctx, one, q[b:b + 1].contiguous(), 1, M, n_new[b:b + 1])
    assert torch.equal(alone[0], out[b])
    ctx.close()


def test_attention_long_context_with_a_sink_and_strided_queries():
    """One token takes nearly all of the weight and thousands share the rest: their part is not lost. Queries are views of a wider
    tensor."""
    Bd, rng = _bd(), np.random.default_rng(11)
    Hq, Hkv, dh, page = 8, 2, 128, 16
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=20000)
    lens = [19000, 16384, 8191]
    kv = _cache(rng, Hkv, dh, page, [L + 1 for L in lens], 1)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    wide, _ = _bf16(rng, (3, Hq * dh + 64), 0.02)
    q = wide[:, 32:32 + Hq * dh]
    for b in range(3):
        pg = kv["block_table"][b, 0]
        kv["k_pages"][pg, :, 0] = R.encode(np.sign(q[b].double().cpu().numpy().reshape(Hkv, Hq // Hkv, dh)[:, 0]))
        kv["k_scales"][pg] = 2.0 ** 4
        kv["v_pages"][pg, :, 0] = 0
        kv["v_scales"][pg] = 2.0 ** -3
    dev = _to_gpu(kv)
    qr = q.double().cpu().numpy().reshape(3, 1, Hq, dh)
    out = torch.zeros((3, 1, Hq, dh), dtype=torch.bfloat16, device="cuda")
    ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), 3, 1, out, ldq=wide.stride(0))
    ref, tol = R.attention(kv, qr, [1, 1, 1], page)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert np.all(err <= tol), float((err / tol).max())
    ctx.close()


def test_attention_rows_do_not_meet_later_rows():
    """What row m + 1 appended is no number: rows up to m give the bits they give without it; a query that is not finite gives NaN."""
    Bd, rng = _bd(), np.random.default_rng(12)
    for Hq, Hkv, dh, M in ((28, 4, 128, 4), (4, 4, 64, 6), (64, 8, 128, 8), (16, 2, 64, 20)):
        page, lens = 16, [0, 5, 44, 300, 1023]
        ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=5 * M, max_K=1, max_ctx=2048)
        kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M)
        kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
        dev = _to_gpu(kv)
        q, _ = _bf16(rng, (5, M, Hq, dh))
        q[3, M - 1, 1, 7] = float("inf")
        good, _ = _attend(Bd, ctx, dev, q, 5, M, None)
        cut = M // 2
        for b, L in enumerate(lens):
            for p in range(L + cut, L + M):
                for w in "kv":
                    dev[w + "_pages"][int(kv["block_table"][b, p // page]), :, p % page] = R.NAN_CODE
        out, _ = _attend(Bd, ctx, dev, q, 5, M, None)
        assert torch.equal(good[:, :cut], out[:, :cut])
        assert torch.isnan(out[:, cut:]).all()
        assert torch.isnan(good[3, M - 1, 1]).all() and torch.isfinite(good[3, M - 1, 2]).all()
        ctx.close()


def test_attention_flags_bad_pages_and_positions():
    Bd, rng = _bd(), np.random.default_rng(13)
    Hq, Hkv, dh, page = 4, 2, 64, 16
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=64)
    kv = _cache(rng, Hkv, dh, page, [40, 30], 8, garbage=False)
    dev = _to_gpu(kv)
    q, qr = _bf16(rng, (2, 2, Hq, dh))
    dev["block_table"][1, 0] = 10 ** 6
    out, st = _attend(Bd, ctx, dev, q, 2, 2, None)
    assert int(st.item()) == Bd.DEV_BAD_PAGE
    dev = _to_gpu(kv)
    dev["seq_lens"][0] = 2 ** 31 - 2                      # beyond every slot: all slots are seen
    out, st = _attend(Bd, ctx, dev, q, 2, 2, None)
    assert int(st.item()) == Bd.DEV_BAD_POS and torch.isfinite(out.float()).all()
    ctx.close()


def test_pool_beyond_32_bit_offsets():
    """Pages whose bytes lie beyond 4 GB of the pool."""
    Bd, rng = _bd(), np.random.default_rng(14)
    Hq, Hkv, dh, page = 8, 4, 128, 16
    num = 2 ** 32 // (Hkv * page * dh) + 40
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=512)
    dev = {w + "_pages": torch.empty((num, Hkv, page, dh), dtype=torch.uint8, device="cuda") for w in "kv"}
    dev.update({w + "_scales": torch.ones((num, Hkv), device="cuda") for w in "kv"})
    pages = [num - 1 - i for i in range(20)]
    dev["block_table"] = torch.tensor([pages], dtype=torch.int32, device="cuda")
    dev["seq_lens"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    x, ref = _bf16(rng, (1, 300, Hkv, dh))
    ctx.fastmtp_kv8_append(x, x, Bd.kv8(dev), 1, 300)
    kv = {"block_table": np.arange(20, dtype=np.int32)[None], "seq_lens": np.zeros(1, np.int32)}
    for w in "kv":
        kv[w + "_pages"] = dev[w + "_pages"][pages].cpu().numpy()
        kv[w + "_scales"] = np.ones((20, Hkv), np.float32)
    want = {k: v.copy() for k, v in kv.items()}
    R.append(want, "k", ref, [300], page)
    for blk in range(19):
        n = min(page, 300 - blk * page)
        assert np.array_equal(kv["k_pages"][blk, :, :n], want["k_pages"][blk, :, :n]), blk
    for w in "kv":
        kv[w + "_scales"] = dev[w + "_scales"][pages].cpu().numpy()
    dev["seq_lens"] += 299
    kv["seq_lens"] = kv["seq_lens"] + 299
    q, qr = _bf16(rng, (1, 1, Hq, dh))
    out, _ = _attend(Bd, ctx, dev, q, 1, 1, None)
    r, tol = R.attention(kv, qr, [1], page)
    assert np.all(np.abs(out.double().cpu().numpy() - r) <= tol)
    back = torch.zeros((1, 8, Hkv, dh), dtype=torch.bfloat16, device="cuda")
    ctx.fastmtp_kv8_read(Bd.kv8(dev), 1, 8, back, torch.zeros_like(back), start=torch.tensor([290], dtype=torch.int32, device="cuda"))
    assert np.array_equal(back.double().cpu().numpy()[0], R.tokens(kv, "k", 0, 298, page)[290:])
    ctx.close()


@pytest.mark.parametrize("garbage", [True, False])
def test_more_rows_than_a_launch_takes_and_other_streams(garbage):
    """Groups of 64 rows; a call on another stream; a captured call replayed with other lengths (which with `garbage` take in slots
    that hold NaN: the same rows have to become NaN)."""
    Bd, rng = _bd(), np.random.default_rng(15)
    Hq, Hkv, dh, page, B, M = 4, 2, 64, 16, 70, 3
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=B * M, max_K=1, max_ctx=512)
    lens = [int(x) for x in rng.integers(0, 300, B)]
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M + 40, garbage)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, qr = _bf16(rng, (B, M, Hq, dh))
    ref, tol = R.attention(kv, qr, [M] * B, page)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.zeros((B, M, Hq, dh), dtype=torch.bfloat16, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, out, stream=side)
    side.synchronize()
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= tol)
    # append + attention captured once, replayed after the lengths moved on
    x, _ = _bf16(rng, (B, M, Hkv, dh))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.fastmtp_kv8_append(x, x, Bd.kv8(dev), B, M)
        ctx.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, out)
    for _ in range(2):
        dev["seq_lens"] += 5
        twin = {k: v.clone() for k, v in dev.items()}
        graph.replay()
        torch.cuda.synchronize()
        o2 = torch.zeros_like(out)
        ctx.fastmtp_kv8_append(x, x, Bd.kv8(twin), B, M)
        ctx.fastmtp_kv8_attention(q, Bd.kv8(twin), B, M, o2)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), o2.view(torch.int16)) and torch.equal(twin["k_pages"], dev["k_pages"])
        assert garbage or torch.isfinite(out.float()).all()
    ctx.close()


def _target_caches(shape, lens, extra, seed):
    """The same random committed K/V as 8-bit caches and, exactly, as bf16 caches."""
    Bd, kvs8, kvs16 = _bd(), [], []
    for layer in range(shape.n_layers):
        rng = np.random.default_rng(seed + layer)
        kv = _cache(rng, shape.n_kv_heads, shape.head_dim, shape.page_size, lens, extra, garbage=False)
        kvs8.append(kv)
        k16 = {"block_table": kv["block_table"], "seq_lens": kv["seq_lens"].copy(), "num_pages": kv["k_pages"].shape[0],
               "max_pages_per_seq": kv["block_table"].shape[1]}
        for w in "kv":
            v = R.TABLE[kv[w + "_pages"]] * kv[w + "_scales"].astype(np.float64)[:, :, None, None]
            k16[w + "_pages"] = I.f32_to_bf16_bits(v.astype(np.float32)).reshape(v.shape)
        kvs16.append(k16)
    return Bd, kvs8, kvs16


@pytest.mark.parametrize("B,M", [(1, 1), (2, 4), (5, 3), (1, 64), (30, 3)])
def test_target_step_over_8_bit_caches(B, M, monkeypatch):
    """Hidden states against the oracle on the same cached values (only the rows of this call enter its cache unrounded, one token in
    hundreds), and layer 0's new codes exactly: the bf16 step's new rows, quantised."""
    monkeypatch.setenv("FMTP_BATCHED_MIN", "1")           # the bf16 step takes the same path: the same bits before the cache
    shape = I.TINY
    lens = [int(x) for x in np.random.default_rng(B * 10 + M).integers(300, 420, B)]
    Bd, kvs8, kvs16 = _target_caches(shape, lens, M, 40 + B)
    W = I.target_weights(shape, 3)
    ctx = Bd.Context(shape, max_rows=B * M, max_K=1, max_ctx=512)
    dW = Bd.to_device(W)
    w, keep = Bd.target_w(dW)
    tok = I.token_ids(9, (B, M), shape.vocab)
    tok_d = torch.from_numpy(tok).cuda()
    d8 = [_to_gpu(k) for k in kvs8]
    d16 = [Bd.to_device(copy_kv(k)) for k in kvs16]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    h8, h16 = (torch.zeros((B, M, shape.d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    logits = torch.zeros((B, M, shape.vocab), dtype=torch.bfloat16, device="cuda")
    arg = torch.zeros((B, M), dtype=torch.int32, device="cuda")
    ctx.fastmtp_target_step_kv8(w, tok_d, [Bd.kv8(k) for k in d8], B, M, h8, logits, arg, st)
    ctx.fastmtp_target_step(w, tok_d, [Bd.kv(k) for k in d16], B, M, h16, None, None, st)
    assert int(st.item()) == 0
    ref, _ = O.target_forward(shape, W, tok, [copy_kv(k) for k in kvs16], want_logits=False)
    close(h8.float().cpu().numpy(), ref, "hidden states")
    assert torch.equal(logits.float().argmax(dim=-1).int(), arg)
    new = {"k": [], "v": []}
    for wname in "kv":
        p16 = d16[0][wname + "_pages"].double().cpu().numpy()
        new[wname] = np.stack([np.stack([p16[kvs16[0]["block_table"][b, (L + m) // 16], :, (L + m) % 16] for m in range(M)])
                               for b, L in enumerate(lens)])
        R.append(kvs8[0], wname, new[wname], [M] * B, 16)
    _same_cache(d8[0], kvs8[0])
    ctx.close()


def test_decoding_over_8_bit_caches_with_log_probabilities():
    """A run as a server makes it: prompt and decoding through loop.Target over 8-bit caches, drafts verified on logits, log
    probabilities of what was emitted."""
    from paper_2509_18362_b200 import loop
    Bd, shape, K = _bd(), I.TINY, 3
    W = I.target_weights(shape, 21)
    ctx = Bd.Context(shape, max_rows=64, max_K=8, max_ctx=256)
    zero = [{"k_pages": np.zeros((17, 2, 16, 64), np.uint8), "v_pages": np.zeros((17, 2, 16, 64), np.uint8),
             "k_scales": np.ones((17, 2), np.float32), "v_scales": np.ones((17, 2), np.float32),
             "block_table": np.random.default_rng(l).permutation(17)[:16].astype(np.int32)[None], "seq_lens": np.zeros(1, np.int32)}
            for l in range(shape.n_layers)]
    prompt = [int(t) for t in I.token_ids(3, (40,), shape.vocab)]
    dW = Bd.to_device(W)
    tgt = loop.Target(ctx, shape, dW, [_to_gpu(k) for k in zero])
    toks = loop.greedy_decode(tgt, prompt, 12)
    assert len(toks) == 12 and int(tgt.status.item()) == 0
    # score three of those tokens at once, from the state before them
    tgt2 = loop.Target(ctx, shape, dW, [_to_gpu(k) for k in zero])
    _, first = loop.prefill(tgt2, prompt)
    assert first == toks[0]
    h, logits, arg = tgt2.step([toks[:K + 1]], want_logits=True)
    drafts = torch.tensor([toks[1:K + 1]], dtype=torch.int32, device="cuda")
    acc, bon = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    ctx.fastmtp_verify_accept(logits, drafts, 1, K, shape.vocab, acc, bon)
    lp, ent = (torch.zeros(K + 1, device="cuda") for _ in range(2))
    ids = torch.zeros((K + 1, 4), dtype=torch.int32, device="cuda")
    tops = torch.zeros((K + 1, 4), device="cuda")
    ctx.fastmtp_logprobs(logits, arg, K + 1, shape.vocab, lp, ent, 4, ids, tops)
    rlp, rent, rids, rtops = R.logprobs(logits[0].double().cpu().numpy(), arg[0].cpu().numpy(), 4)
    assert np.array_equal(ids.cpu().numpy(), rids) and torch.equal(ids[:, 0], arg[0])
    for got, ref in ((lp, rlp), (ent, rent), (tops, rtops)):
        assert np.abs(got.double().cpu().numpy() - ref).max() <= 2e-5 + 2.0 ** -23 * np.abs(ref).max()
    n = int(acc.item())
    assert all(int(arg[0, j]) == toks[1 + j] for j in range(n))
    ctx.close()


def test_refusals():
    Bd = _bd()
    ctx = Bd.Context(_shape(4, 2, 64, 16), max_rows=8, max_K=1, max_ctx=64)
    kv = _to_gpu(_cache(np.random.default_rng(0), 2, 64, 16, [3], 8))
    x = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    o = torch.zeros((4, 4, 4, 64), dtype=torch.bfloat16, device="cuda")
    ok = Bd.kv8(kv)
    null = Bd.kv8(kv)
    null.v_scales = None
    huge = Bd.kv8(kv)
    huge.num_pages = 2 ** 31 - 1
    odd = Bd.kv8(kv)
    odd.k_pages = kv["k_pages"].data_ptr() + 8

    def code(f, *a, **k):
        with pytest.raises(Bd.FastMTPError) as e:
            f(*a, **k)
        return e.value.code

    ap, at, rd = ctx.fastmtp_kv8_append, ctx.fastmtp_kv8_attention, ctx.fastmtp_kv8_read
    for c in (lambda kv_: code(ap, x, x, kv_, 1, 1), lambda kv_: code(at, x, kv_, 1, 1, o), lambda kv_: code(rd, kv_, 1, 4, x, x)):
        assert c(null) == -1 and c(huge) == -2 and c(odd) == -1
    assert code(ap, None, x, ok, 1, 1) == -1 and code(ap, x, x, ok, 0, 1) == -1 and code(ap, x, x, ok, 1, 0) == -1
    assert code(ap, x, x, ok, 1, 1, ld=127) == -1 and code(ap, x, x, ok, 1, 2, ld=132) == -1 and code(ap, x[1:], x, ok, 1, 1) == -1
    assert code(at, x, ok, 1, 1, None) == -1 and code(at, x, ok, 1, 65, o) == -2 and code(at, x, ok, 9, 1, o) == -2
    assert code(at, x, ok, 1, 1, o, ldq=248) == -1 and code(at, x[4:], ok, 1, 1, o) == -1 and code(at, x, ok, -1, 1, o) == -1
    assert code(rd, ok, 1, 0, x, x) == -1 and code(rd, ok, 1, 4, None, x) == -1 and code(rd, ok, 1, 4, x[2:], x) == -1
    launches = ctx.launch_count
    at(x, ok, 1, 1, o)
    assert ctx.launch_count > launches
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,page,M", [(16, 2, 128, 16, 5), (64, 8, 128, 48, 16), (8, 8, 128, 16, 64), (28, 4, 128, 32, 64),
                                              (8, 1, 128, 5, 9), (8, 2, 64, 16, 17)])
def test_attention_of_many_pairs_against_64_bits(Hq, Hkv, dh, page, M):
    """40, 128, 64 and 448 pairs per KV head in tiles of 128; blocks that are no whole 16 tokens and head dimension 64, which have none."""
    test_attention_against_64_bits(Hq, Hkv, dh, page, M)


@pytest.mark.parametrize("Hq,Hkv,dh,M", [(8, 1, 128, 1), (8, 1, 128, 4), (8, 1, 128, 8), (8, 1, 64, 8)])
def test_attention_with_scores_and_scales_that_climb(Hq, Hkv, dh, M):
    """Every block's scores lie far above the ones before and its V scale is larger or far smaller: the reference and the largest
    V scale move many times within a chunk, down to a scale that counts as nothing."""
    Bd, rng = _bd(), np.random.default_rng(31 + M + dh)
    page, L = 16, 700
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=8, max_K=1, max_ctx=1024)
    kv = _cache(rng, Hkv, dh, page, [L + M], M, garbage=False)
    kv["seq_lens"] = np.asarray([L], dtype=np.int32)
    q = torch.ones((1, M, Hq, dh), dtype=torch.bfloat16, device="cuda") * 2.0 ** -6
    for i, pg in enumerate(kv["block_table"][0][:(L + M + page - 1) // page]):
        kv["k_pages"][pg] = R.encode(np.full((Hkv, page, dh), 1.0) + 0.25 * rng.integers(0, 2, (Hkv, page, dh)))
        kv["k_scales"][pg] = 0.5 + 0.75 * i
        kv["v_scales"][pg] = (2.0 ** (i / 2 - 10), 1.5, 2.0 ** -90)[i % 3]
    dev = _to_gpu(kv)
    out, st = _attend(Bd, ctx, dev, q, 1, M, None)
    for w in "kv":
        kv[w + "_scales"] = dev[w + "_scales"].cpu().numpy()
    ref, tol = R.attention(kv, q.double().cpu().numpy(), [M], page)
    err = np.abs(out.double().cpu().numpy() - ref)
    assert np.all(err <= tol), float((err / tol).max())
    assert int(st.item()) == 0
    ctx.close()


@pytest.mark.parametrize("Hq,Hkv,dh,M", [(28, 4, 128, 1), (28, 4, 128, 4), (64, 8, 128, 8), (28, 4, 128, 64), (16, 2, 64, 20)])
def test_attention_puts_a_value_that_is_no_number_where_it_is_seen(Hq, Hkv, dh, M):
    """One dimension of one token's value, committed or new: that dimension of the rows that see it, and no other bit."""
    Bd, rng = _bd(), np.random.default_rng(41 + M)
    page, lens = 16, [0, 70, 600]
    ctx = Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=3 * M, max_K=1, max_ctx=1024)
    kv = _cache(rng, Hkv, dh, page, [L + M for L in lens], M)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, _ = _bf16(rng, (3, M, Hq, dh))
    good, _ = _attend(Bd, ctx, dev, q, 3, M, None)
    want = good.clone()
    g = Hq // Hkv
    for b, L in enumerate(lens):
        for p, kvh, d in ((L + M // 2, 0, 3), (L + M - 1, Hkv - 1, dh - 2)) + (((L - 30, 1, 17),) if L else ()):
            dev["v_pages"][int(kv["block_table"][b, p // page]), kvh, p % page, d] = R.NAN_CODE | (0x80 if d == 3 else 0)
            want[b, max(0, p - L):, kvh * g:(kvh + 1) * g, d] = float("nan")
    out, _ = _attend(Bd, ctx, dev, q, 3, M, None)
    assert torch.equal(torch.isnan(want), torch.isnan(out))
    assert torch.equal(want.nan_to_num(7.0), out.nan_to_num(7.0))
    ctx.close()


def test_tiles_of_pairs_in_graphs_beside_other_streams_and_with_bad_pages():
    """140 pairs per KV head: a captured call replayed at other lengths, two contexts on two streams at once, a page that does not
    exist."""
    Bd, rng = _bd(), np.random.default_rng(51)
    Hq, Hkv, dh, page, B, M = 28, 4, 128, 16, 5, 20
    lens = [0, 33, 700, 1500, 64]
    ctxs = [Bd.Context(_shape(Hq, Hkv, dh, page), max_rows=B * M, max_K=1, max_ctx=2048) for _ in range(2)]
    kv = _cache(rng, Hkv, dh, page, [L + M + 70 for L in lens], 0, garbage=False)
    kv["seq_lens"] = np.asarray(lens, dtype=np.int32)
    dev = _to_gpu(kv)
    q, _ = _bf16(rng, (B, M, Hq, dh))
    want, st = _attend(Bd, ctxs[0], dev, q, B, M, None)
    assert int(st.item()) == 0
    outs = [torch.zeros_like(want) for _ in ctxs]
    streams = [torch.cuda.Stream() for _ in ctxs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, o in zip(ctxs, streams, outs):
            c.fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctxs[0].fastmtp_kv8_attention(q, Bd.kv8(dev), B, M, out)
    for step in (3, 64):
        dev["seq_lens"] += step
        graph.replay()
        eager, _ = _attend(Bd, ctxs[1], dev, q, B, M, None)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.isfinite(out.float()).all()
    dev["block_table"][2, 7] = -5
    bad, st = _attend(Bd, ctxs[0], dev, q, B, M, None)
    assert int(st.item()) == Bd.DEV_BAD_PAGE
    keep = [0, 1, 3, 4]
    assert torch.equal(bad[keep], out[keep])
    for c in ctxs:
        c.close()
