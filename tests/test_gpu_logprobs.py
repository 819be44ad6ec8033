"""fastmtp_logprobs against float64: ids exactly, values within bounds.

The bound: terms e^(x - m) are off by 2^-22 and by the rounding of (x - m) log2(e) (2^-24 of it, which a term e^d |d| <= 0.37 keeps
below 2^-23 of the largest), sums by 2^-24 for each of at most 330 additions in a row (a thread's share of 152064 values in
two accumulators, then a tree): 2e-5 of S, so 2e-5 of its logarithm; the same of T / S, which is at most the entropy plus ln S. Results are
rounded to fp32 (2^-24)."""
import numpy as np
import pytest
import torch

from . import kv8_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_2509_18362_b200 import binding as Bd
    from paper_2509_18362_b200 import inputs as I
    c = Bd.Context(I.TINY, max_rows=8, max_K=1, max_ctx=64)
    yield c
    c.close()


def _run(ctx, x, tok, top, V, ld=None, stream=None):
    rows = len(tok)
    lp, ent = (torch.full((rows,), 5.0, device="cuda") for _ in range(2))
    ids = torch.full((rows, top), -3, dtype=torch.int32, device="cuda")
    tops = torch.full((rows, top), 5.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.fastmtp_logprobs(x, torch.as_tensor(tok, dtype=torch.int32).cuda(), rows, V, lp, ent, top, ids if top else None, tops if top else None,
                         dev_status=st, ld=ld, stream=stream)
    torch.cuda.synchronize()
    return lp.double().cpu().numpy(), ent.double().cpu().numpy(), ids.cpu().numpy(), tops.double().cpu().numpy(), int(st.item())


def _near(got, ref, what):
    fin = np.isfinite(ref)
    assert np.array_equal(np.isfinite(got), fin) and np.array_equal(got[~fin], ref[~fin]), (what, got, ref)
    err = np.abs(got[fin] - ref[fin])
    assert np.all(err <= 2e-5 + 2.0 ** -23 * np.abs(ref[fin])), (what, err.max())


def _check(ctx, x, tok, top, V=None, ld=None):
    """x: [rows, >= V] tensor on the GPU."""
    V = x.shape[1] if V is None else V
    lp, ent, ids, tops, st = _run(ctx, x, tok, top, V, ld)
    rlp, rent, rids, rtops = R.logprobs(x[:, :V].double().cpu().numpy(), tok, top)
    assert np.array_equal(ids, rids), np.argwhere(ids != rids)[:5]
    _near(lp, rlp, "logprob")
    _near(tops, rtops, "tops")
    err = np.abs(ent - rent)
    assert np.all(err <= 4e-5 * (1 + rent)), err.max()
    return st


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,V,top", [
    (1, 1, 1), (2, 7, 7), (3, 8, 0), (3, 9, 2), (5, 33, 32), (1, 2047, 20), (4, 2049, 5), (300, 1000, 8), (4, 152064, 20), (37, 16385, 32),
    (260, 4099, 1), (1, 1000001, 3), (64, 20000, 32),
])
def test_against_64_bits(ctx, f32, rows, V, top):
    """Rows at every alignment, shorter and longer than a slice; a second call finds the scratch as the first one did."""
    rng = np.random.default_rng(rows * 7919 + V)
    x = rng.standard_normal((rows, V + rows % 3)).astype(np.float32) * 3
    x[::2, rng.integers(0, V)] += 9
    t = torch.from_numpy(x).cuda()
    t = t if f32 else t.to(torch.bfloat16)
    tok = rng.integers(0, V, rows)
    for _ in range(2):
        assert _check(ctx, t, tok, top, V, t.stride(0)) == 0


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_ties_masks_and_values_that_are_no_numbers(ctx, f32, V):
    rng = np.random.default_rng(V)
    lowest = float(torch.finfo(torch.float32 if f32 else torch.bfloat16).min)
    x = (np.round(rng.standard_normal((16, V)) * 2) / 2).astype(np.float32)           # many ties
    x[1] = 0.25                                            # all equal
    x[2] = np.sort(x[2])                                   # ascending: every slice beats the ones before
    x[3] = -np.sort(-x[3])
    x[4] = -np.inf
    x[4, V // 2] = -3.0                                    # one id is left
    x[5] = lowest
    x[5, [V - 1, 3]] = 1.0
    x[6] = lowest                                          # masked altogether by the type's lowest number
    x[6, 2] = -np.inf
    x[7] = np.nan
    x[7, 5:30] = np.arange(25)[::-1]
    x[8, [7, V - 2]] = np.inf                              # two infinite maxima share
    x[9] = 0.0
    x[9, ::2] = -0.0
    x[10, :] = -1e4
    x[10, 9] = 1e4
    x[11] = 2.0 ** 100
    x[11, 1] = -(2.0 ** 100)
    x[12] = -np.inf
    x[13] = np.nan
    x[14, ::3] = np.nan
    x[15] = -(2.0 ** 110) * (1 + np.arange(V) % 5)
    t = torch.from_numpy(x).cuda()
    t = t if f32 else t.to(torch.bfloat16)
    from paper_2509_18362_b200 import binding as Bd
    tok = np.array([0, 3, 1, 1, V // 2, 3, 7, 6, 7, 8, 9, 0, 0, 4, 3, 5])
    for top in (0, 1, 20, 32):
        assert _check(ctx, t, tok, top) == Bd.DEV_ALL_NAN
    tok = np.array([V - 1] * 16)
    _check(ctx, t, tok, 5)


@pytest.mark.parametrize("spread", [1, 3, 64])
def test_every_element_of_a_few_threads_is_a_candidate(ctx, spread):
    """The largest values crowd into the vectors that few threads hold, more of them than are asked for, in every slice."""
    V = 70000
    x = torch.zeros((3, V), device="cuda")
    idx = torch.arange(V, device="cuda")
    hot = (idx // 8) % 256 < spread
    x[:, hot] = 5 + (idx[hot] % 97).float() / 97
    x[1] += idx / V                                        # and the later the larger
    x[2] = torch.where(hot, 6.0, x[2])
    _check(ctx, x.to(torch.bfloat16), np.array([0, 9, 2049]), 32)
    _check(ctx, x, np.array([0, 9, 2049]), 20)


def test_outputs_may_be_left_out_and_bad_tokens_are_flagged(ctx):
    from paper_2509_18362_b200 import binding as Bd
    x = torch.randn((6, 500), device="cuda", dtype=torch.bfloat16)
    ent = torch.zeros(6, device="cuda")
    ctx.fastmtp_logprobs(x, None, 6, 500, None, ent)
    _, rent, _, _ = R.logprobs(x.double().cpu().numpy(), [0] * 6, 1)
    assert np.abs(ent.double().cpu().numpy() - rent).max() <= 4e-5 * (1 + rent.max())
    lp, _, _, _, st = _run(ctx, x, [0, 500, -1, 3, 2 ** 31 - 1, 499], 0, 500)
    rlp, _, _, _ = R.logprobs(x.double().cpu().numpy(), [0, 0, 0, 3, 0, 499], 1)
    _near(lp, rlp, "clamped")
    assert st == Bd.DEV_BAD_TOKEN


def test_same_bits_again_on_another_stream_and_in_a_graph(ctx):
    x = torch.randn((9, 30011), device="cuda", dtype=torch.bfloat16) * 2
    tok = np.arange(9)
    a = _run(ctx, x, tok, 7, 30011)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = _run(ctx, x, tok, 7, 30011, stream=side)
    for u, v in zip(a, b):
        assert np.array_equal(u, v)
    lp = torch.zeros(9, device="cuda")
    t = torch.from_numpy(tok.astype(np.int32)).cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.fastmtp_logprobs(x, t, 9, 30011, lp)
    x.copy_(torch.randn((9, 30011), device="cuda"))
    graph.replay()
    c = _run(ctx, x, tok, 7, 30011)
    assert np.array_equal(lp.double().cpu().numpy(), c[0])


def test_refusals(ctx):
    from paper_2509_18362_b200 import binding as Bd
    x = torch.zeros((4, 64), device="cuda", dtype=torch.bfloat16)
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    o = torch.zeros(4, device="cuda")
    ids = torch.zeros((4, 64), dtype=torch.int32, device="cuda")

    def code(*a, **k):
        with pytest.raises(Bd.FastMTPError) as e:
            ctx.fastmtp_logprobs(*a, **k)
        return e.value.code

    assert code(None, t, 4, 64, o) == -1 and code(x, None, 4, 64, o) == -1 and code(x, t, 0, 64, o) == -1 and code(x, t, 4, 0, o) == -1
    assert code(x, t, 4, 64, o, None, 5) == -1 and code(x, t, 4, 64, o, None, -1, ids) == -1 and code(x, t, 4, 64, o, None, 33, ids) == -2
    assert code(x, t, 4, 16, o, None, 17, ids) == -1 and code(x, t, 4, 64, o, ld=63) == -1 and code(x, t, 4097, 1, o) == -2
    assert code(x.half(), t, 4, 64, o) == -3
    ctx.fastmtp_logprobs(x, t, 4, 64, o)
    assert np.allclose(o.cpu().numpy(), -np.log(64), atol=2e-5)
