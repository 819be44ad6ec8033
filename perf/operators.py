"""The library's operators around an 8-bit cache and a verification's answer, as cases to be timed and compared.

Four entry points: fastmtp_kv8_append (quantising K/V rows into a paged e4m3 cache with one scale for each block of tokens and
head), fastmtp_kv8_read (reading such a cache back), fastmtp_kv8_attention (attention over it, from one token per sequence
to a chunk of a prompt) and fastmtp_logprobs (log probability of given tokens, entropy, top alternatives). A case is one
call. Head layouts are those of the package's shapes (28 query / 4 KV heads of 128, 4 / 2 of 64) and generic ones; contexts,
batches and rows are those of the package's benchmark and tests, vocabularies up to its 152064. With `own` unset the
operators are computed from elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

E4M3 = torch.float8_e4m3fn
HEADS = [(28, 4, 128), (32, 8, 128), (16, 16, 64), (4, 2, 64), (8, 1, 128), (64, 8, 128)]


def _kv(name, op, B, M, lo, hi, heads=(28, 4, 128), page=16, short=False):
    c = {"op": op, "B": B, "M": M, "ctx_min": lo, "ctx_max": hi, "Hq": heads[0], "Hkv": heads[1], "dh": heads[2], "page": page,
         "short": short}
    return dict(c, name=name) if name else c


def _lp(name, rows, V, top, f32=False, pad=0):
    c = {"op": "logprobs", "rows": rows, "V": V, "top": top, "f32": f32, "pad": pad}
    return dict(c, name=name) if name else c


def listed():
    return [
        # every sequence of a ragged batch decodes one token: its K/V row enters a partly filled block
        _kv("append_decode_b37", "append", 37, 1, 100, 1500),
        # prompts enter the cache: 16 of up to 4096 tokens each
        _kv("append_prompt_b16", "append", 16, 4096, 0, 900, short=True),
        # one request's cache goes back to 16 bits
        _kv("read_b1", "read", 1, 0, 2048, 2048),
        # a batch's ragged caches do (another head layout, longer blocks)
        _kv("read_b32_ragged", "read", 32, 0, 512, 8192, heads=(32, 8, 128), page=32),
        # one request being decoded: all latency
        _kv("attn_decode_b1", "attention", 1, 1, 2048, 2048),
        # a full batch with ragged long contexts
        _kv("attn_decode_b64_ragged", "attention", 64, 1, 512, 8192),
        # two requests with very long contexts
        _kv("attn_decode_b2_long", "attention", 2, 1, 50000, 60000, heads=(32, 8, 128)),
        # scoring of three drafts per request; some requests have fewer, some none
        _kv("attn_score_b17", "attention", 17, 4, 1, 4100, short=True),
        # chunks of 64 prompt tokens
        _kv("attn_prompt64_b4", "attention", 4, 64, 3500, 4200),
        # log probabilities of one request's verification
        _lp("logprobs_r4", 4, 152064, 5),
        # of a full batch's, with the alternatives a server returns
        _lp("logprobs_r256", 256, 152064, 20),
        # of draft tokens over a compressed vocabulary, fp32 logits with padded rows
        _lp("logprobs_f32_r75", 75, 32001, 8, f32=True, pad=31),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    op = rng.choice(["append", "read", "attention", "attention", "logprobs"])
    if op == "logprobs":
        V = _log_int(rng, 1000, 152064)
        rows = _log_int(rng, 1, min(1024, 256 * 152064 // V))
        return _lp(None, rows, V, rng.choice([0, 1, 5, 20, 32]), f32=rng.random() < 0.3 and rows * V < 128 * 152064,
                   pad=rng.choice([0, 0, 1, 64]))
    heads, page = rng.choice(HEADS), rng.choice([16, 16, 16, 32, 64, 8, 5])
    token = 2 * heads[1] * heads[2]                                      # values of a token
    if op == "append":
        B = _log_int(rng, 1, 64)
        M = rng.randint(1, 8) if rng.random() < 0.5 else _log_int(rng, 9, 4096)
        M = max(1, min(M, 65536 * 1024 // token // B))
        hi = _log_int(rng, 1, 2000)
        return _kv(None, op, B, M, rng.randint(0, hi), hi, heads, page, rng.random() < 0.5)
    if op == "read":
        B = _log_int(rng, 1, 32)
        hi = min(_log_int(rng, 16, 8192), 270_000_000 // token // B)
        return _kv(None, op, B, 0, rng.randint(0, hi), hi, heads, page, rng.random() < 0.5)
    B, kind = _log_int(rng, 1, 64), rng.random()
    M = 1 if kind < 0.5 else rng.randint(2, 8) if kind < 0.85 else rng.randint(9, 64)
    hi = min(_log_int(rng, 1, 65536), 270_000_000 // token // B, int(1.4e10 / (4 * heads[0] * heads[2] * M * B)))
    return _kv(None, op, B, M, rng.randint(hi // 8, hi), hi, heads, page, rng.random() < 0.4)


# ---- sizes that belong to a case (the same for every seed)

def _lengths(case):
    """Committed tokens of every sequence, and the rows of this call that count."""
    r = random.Random(case["B"] * 1000003 + case["ctx_max"])
    L = [r.randint(case["ctx_min"], case["ctx_max"]) for _ in range(case["B"])]
    M = case["M"]
    n = [r.randint(0, M) if case["short"] else M for _ in range(case["B"])]
    n[r.randrange(case["B"])] = M
    return L, n


def work(case):
    if case["op"] == "logprobs":
        size = 4 if case["f32"] else 2
        return {"bytes": case["rows"] * (case["V"] * size + 12 + 8 * case["top"]), "flops": 4 * case["rows"] * case["V"]}
    L, n = _lengths(case)
    token = 2 * case["Hkv"] * case["dh"]
    if case["op"] == "append":
        return {"bytes": sum(n) * token * 3 + sum(1 for x in n if x) * 2 * case["Hkv"] * 4, "flops": 2 * sum(n) * token}
    if case["op"] == "read":
        return {"bytes": sum(L) * token * 3, "flops": sum(L) * token}
    seen = sum(L[b] + n[b] for b in range(len(L)) if n[b])
    pairs = sum(n[b] * L[b] + n[b] * (n[b] + 1) // 2 for b in range(len(L)))
    return {"bytes": seen * token + sum(n) * case["Hq"] * case["dh"] * 4, "flops": 4 * case["Hq"] * case["dh"] * pairs}


# ---- inputs

def _codes(g, shape, device):
    """A pool as a cache fills it: values with a spread over channels and tokens, quantised block by block."""
    pages, hkv, page, dh = shape
    x = torch.randn(shape, generator=g, device=device)
    x *= torch.exp2(torch.randn((1, hkv, 1, dh), generator=g, device=device))
    x *= torch.exp2(0.5 * torch.randn((pages, 1, page, 1), generator=g, device=device))
    s = _scale_for(x.abs().amax(dim=(2, 3)))
    return (x / s[:, :, None, None]).to(E4M3), s


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev).manual_seed(int(seed) * 2654435761 % (1 << 62) + 17)
    st = {"case": case}
    if case["op"] == "logprobs":
        R, V, ld = case["rows"], case["V"], case["V"] + case["pad"]
        x = torch.randn((R, ld), generator=g, device=dev) * 2
        # every other row has a clear favourite, as most positions of a text have
        peak = torch.randint(0, V, (R,), generator=g, device=dev)
        x[torch.arange(0, R, 2, device=dev), peak[::2]] += 10 + 4 * torch.rand(((R + 1) // 2,), generator=g, device=dev)
        x = x if case["f32"] else x.to(torch.bfloat16)
        toks = torch.where(torch.rand((R,), generator=g, device=dev) < 0.7, peak, torch.randint(0, V, (R,), generator=g, device=dev))
        st.update(logits=x[:, :V], tokens=toks.to(torch.int32))
        st["logprob"] = torch.zeros(R, device=dev)
        st["entropy"] = torch.zeros(R, device=dev)
        st["ids"] = torch.zeros((R, case["top"]), dtype=torch.int32, device=dev)
        st["tops"] = torch.zeros((R, case["top"]), device=dev)
    else:
        B, M, Hq, Hkv, dh, page = (case[k] for k in ("B", "M", "Hq", "Hkv", "dh", "page"))
        L, n = _lengths(case)
        per = [max(1, -(-(l + M) // page)) for l in L]
        perm = torch.randperm(sum(per) + 3, generator=g, device=dev).tolist()
        table = torch.full((B, max(per)), -1, dtype=torch.int32)
        at = 0
        for b, p in enumerate(per):
            table[b, :p] = torch.tensor(perm[at:at + p], dtype=torch.int32)
            at += p
        st["k_pages"], st["k_scales"] = _codes(g, (len(perm), Hkv, page, dh), dev)
        st["v_pages"], st["v_scales"] = _codes(g, (len(perm), Hkv, page, dh), dev)
        st["block_table"] = table.to(dev)
        st["seq_lens"] = torch.tensor(L, dtype=torch.int32, device=dev)
        st["n_new"] = torch.tensor(n, dtype=torch.int32, device=dev)
        if case["op"] == "read":
            st["out_k"] = torch.zeros((B, max(L), Hkv, dh), dtype=torch.bfloat16, device=dev)
            st["out_v"] = torch.zeros_like(st["out_k"])
        else:
            # rows of a fused projection: query heads, key heads, value heads side by side
            wide = (Hq + 2 * Hkv) * dh
            rows = torch.randn((B * M, wide), generator=g, device=dev)
            rows *= torch.exp2(torch.randn((1, wide), generator=g, device=dev))
            st["rows"] = rows.to(torch.bfloat16)
            st["out"] = torch.zeros((B, M, Hq, dh), dtype=torch.bfloat16, device=dev)
    if own:
        from paper_2509_18362_b200 import binding as Bd
        from paper_2509_18362_b200 import inputs as I
        if case["op"] == "logprobs":
            st["ctx"] = Bd.Context(I.TINY, max_rows=8, max_K=1, max_ctx=64)
        else:
            shape = I.Shape(d=512, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=dh, ffn=512, vocab=1024, n_layers=1, page_size=page)
            rows = B * M if case["op"] == "attention" else 8
            st["ctx"] = Bd.Context(shape, max_rows=rows, max_K=1, max_ctx=max(L) + M + 1)
            st["kv8"] = Bd.kv8(st)
        st["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    return st


# ---- the operators in their plain form

def _scale_for(amax):
    """Smallest power of two s (2^-120 at least) with amax <= 448 s."""
    frac, exp = torch.frexp(amax)                                        # amax = frac * 2^exp, frac in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(frac > 0.875, exp - 8, exp - 9).clamp(min=-120)
    return torch.ldexp(torch.ones_like(amax), e)


def _take(pages, index):
    return pages.view(torch.uint8)[index].view(E4M3)


def _append_one(pages, scales, x, st, case):
    """x [B, M, Hkv, dh]: quantises the rows that count into their blocks."""
    B, M, Hkv, dh = x.shape
    page, dev = case["page"], x.device
    L, n = st["seq_lens"].long(), st["n_new"].long()
    nb = (M + page - 1) // page + 1                                      # blocks that M rows can touch
    blk = (L // page)[:, None] + torch.arange(nb, device=dev)
    pos = blk[:, :, None] * page + torch.arange(page, device=dev)        # [B, nb, page]
    new = (pos >= L[:, None, None]) & (pos < (L + n)[:, None, None])
    old = pos < L[:, None, None]
    b, i = torch.nonzero(new.any(dim=2), as_tuple=True)                  # the blocks that get new tokens
    new, old = new[b, i][:, None, :, None], old[b, i][:, None, :, None]
    ids = st["block_table"].long()[b, blk[b, i]]
    row = (pos[b, i] - L[b, None]).clamp(0, M - 1)
    rows = x[b[:, None], row].float().transpose(1, 2)                    # [blocks, Hkv, page, dh]
    codes, s_old = _take(pages, ids), scales[ids]
    counted = torch.where(new & torch.isfinite(rows), rows.abs(), 0.0)
    need = _scale_for(counted.amax(dim=(2, 3)))
    s_new = torch.where(old.any(dim=2)[:, :, 0], torch.maximum(need, s_old), need)
    fresh = (rows / s_new[:, :, None, None]).clamp(-448, 448).to(E4M3)
    again = (codes.float() * (s_old / s_new)[:, :, None, None]).to(E4M3)
    pick = lambda c, a, z: torch.where(c, a.view(torch.uint8), z.view(torch.uint8))  # noqa: E731
    pages.view(torch.uint8)[ids] = pick(new, fresh, pick(old, again, codes).view(E4M3))
    scales[ids] = s_new


def _dense(pages, scales, st):
    """[B, tokens, Hkv, dh] in 32 bits; what lies behind a sequence's last block is block 0."""
    t = st["block_table"].long().clamp(min=0)
    x = _take(pages, t).float() * scales[t][:, :, :, None, None]         # [B, blocks, Hkv, page, dh]
    return x.transpose(2, 3).flatten(1, 2)


def _plain(st):
    case = st["case"]
    if case["op"] == "logprobs":
        x = st["logits"].float()
        V, top = case["V"], case["top"]
        m = x.amax(dim=1, keepdim=True)
        d = x - m
        p = torch.exp(d)
        S = p.sum(dim=1, keepdim=True)
        lse = torch.log(S)
        logprob = d.gather(1, st["tokens"].long()[:, None]) - lse
        entropy = lse - torch.where(p > 0, p * d, 0.0).sum(dim=1, keepdim=True) / S
        # (value, id) as one whole number: the larger value first, then the lower id
        bits = (x + 0.0).contiguous().view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7fffffff), bits) * (1 << 20) + (V - 1 - torch.arange(V, device=x.device))
        best = torch.topk(key, top, dim=1, sorted=True).values
        ids = V - 1 - (best & ((1 << 20) - 1))
        return {"logprob": logprob[:, 0], "entropy": entropy[:, 0], "ids": ids.to(torch.int32), "tops": d.gather(1, ids) - lse}
    B, M, Hq, Hkv, dh = (case[k] for k in ("B", "M", "Hq", "Hkv", "dh"))
    L = st["seq_lens"].long()
    if case["op"] == "read":
        T = st["out_k"].shape[1]
        seen = (torch.arange(T, device=L.device) < L[:, None])[:, :, None, None]
        pair = [torch.where(seen, _dense(st[w + "_pages"], st[w + "_scales"], st)[:, :T].to(torch.bfloat16), st["out_" + w]) for w in ("k", "v")]
        return {"k": pair[0], "v": pair[1]}
    rows = st["rows"].view(B, M, Hq + 2 * Hkv, dh)
    if case["op"] == "append":
        _append_one(st["k_pages"], st["k_scales"], rows[:, :, Hq:Hq + Hkv], st, case)
        _append_one(st["v_pages"], st["v_scales"], rows[:, :, Hq + Hkv:], st, case)
        return {k: st[k] for k in ("k_pages", "v_pages", "k_scales", "v_scales")}
    q = rows[:, :, :Hq].float().reshape(B, M, Hkv, Hq // Hkv, dh)
    k, v = (_dense(st[w + "_pages"], st[w + "_scales"], st) for w in ("k", "v"))
    s = torch.einsum("bmhgd,bthd->bhgmt", q, k) / math.sqrt(dh)
    pos = torch.arange(k.shape[1], device=q.device)
    seen = pos <= L[:, None, None] + torch.arange(M, device=q.device)[:, None]                # [B, M, tokens]
    s = torch.where(seen[:, None, None], s, -math.inf)
    p = torch.exp(s - s.amax(dim=-1, keepdim=True))
    o = torch.einsum("bhgmt,bthd->bmhgd", p, v) / p.sum(dim=-1).permute(0, 3, 1, 2)[..., None]
    counts = (torch.arange(M, device=q.device) < st["n_new"][:, None])[:, :, None, None]
    return torch.where(counts, o.reshape(B, M, Hq, dh).to(torch.bfloat16), st["out"])


# ---- the framework's

def run(st):
    if not own:
        return _plain(st)
    case, ctx = st["case"], st["ctx"]
    if case["op"] == "logprobs":
        ctx.fastmtp_logprobs(st["logits"], st["tokens"], case["rows"], case["V"], st["logprob"], st["entropy"], case["top"],
                             st["ids"], st["tops"], dev_status=st["status"], ld=st["logits"].stride(0))
        return {k: st[k] for k in ("logprob", "entropy", "ids", "tops")}
    B, M, Hq, Hkv, dh = (case[k] for k in ("B", "M", "Hq", "Hkv", "dh"))
    if case["op"] == "read":
        ctx.fastmtp_kv8_read(st["kv8"], B, st["out_k"].shape[1], st["out_k"], st["out_v"], dev_status=st["status"])
        return {"k": st["out_k"], "v": st["out_v"]}
    rows = st["rows"]
    ld = rows.stride(0)
    n_new = st["n_new"] if case["short"] else None
    if case["op"] == "append":
        ctx.fastmtp_kv8_append(rows[:, Hq * dh:], rows[:, (Hq + Hkv) * dh:], st["kv8"], B, M, n_new=n_new, dev_status=st["status"],
                               ld=ld)
        return {k: st[k] for k in ("k_pages", "v_pages", "k_scales", "v_scales")}
    ctx.fastmtp_kv8_attention(rows, st["kv8"], B, M, st["out"], n_new=n_new, dev_status=st["status"], ldq=ld)
    return st["out"]


# ---- the definition in 64 bits, written apart from the forms above

def _round_e4m3(x):
    """Nearest e4m3 number (ties to even) of doubles within +-448: steps of 2^-9 below 2^-6, of an eighth of the binade above."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step                                  # torch.round: halves to even


def _pow2_over(a):
    e = torch.ceil(torch.log2((a / 448).clamp(min=2.0 ** -120)))
    s = torch.exp2(e)
    return torch.where(a <= 448 * (s / 2), torch.where(e > -120, s / 2, s), torch.where(a > 448 * s, s * 2, s))


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "logprobs":
        x = st["logits"].double()
        order = torch.sort(x, dim=1, descending=True, stable=True)       # equal values stay in the order of their ids
        lse = torch.logsumexp(x, dim=1, keepdim=True)
        ids = order.indices[:, :case["top"]]
        p = torch.softmax(x, dim=1)
        return {"logprob": (x.gather(1, st["tokens"].long()[:, None]) - lse)[:, 0], "entropy": torch.special.entr(p).sum(dim=1),
                "ids": ids.to(torch.int32), "tops": x.gather(1, ids) - lse}
    B, M, Hq, Hkv, dh, page = (case[k] for k in ("B", "M", "Hq", "Hkv", "dh", "page"))
    L, n = _lengths(case)
    table = st["block_table"].tolist()

    def tokens(which, b, count):
        """The first `count` tokens of a sequence's cache as doubles [count, Hkv, dh]."""
        ids = torch.tensor(table[b][:-(-count // page)], device="cuda", dtype=torch.long)
        v = st[which + "_pages"].view(torch.uint8)[ids].view(E4M3).double() * st[which + "_scales"][ids].double()[:, :, None, None]
        return v.permute(0, 2, 1, 3).reshape(-1, Hkv, dh)[:count]

    if case["op"] == "read":
        out = {w: torch.zeros(st["out_k"].shape, dtype=torch.float64, device="cuda") for w in ("k", "v")}
        for b in range(B):
            for w in ("k", "v"):
                if L[b]:
                    out[w][b, :L[b]] = tokens(w, b, L[b])
        return out
    rows = st["rows"].double().view(B, M, Hq + 2 * Hkv, dh)
    if case["op"] == "append":
        out = {w: st[w].double() for w in ("k_pages", "v_pages", "k_scales", "v_scales")}
        for b in range(B):
            if n[b] == 0:
                continue
            first, end = L[b] // page, L[b] + n[b]
            count = -(-end // page) - first
            ids = torch.tensor(table[b][first:first + count], device="cuda", dtype=torch.long)
            lead = L[b] - first * page
            for w, h0 in (("k", Hq), ("v", Hq + Hkv)):
                x = torch.zeros((count * page, Hkv, dh), dtype=torch.float64, device="cuda")
                x[lead:lead + n[b]] = rows[b, :n[b], h0:h0 + Hkv]
                x = x.view(count, page, Hkv, dh).permute(0, 2, 1, 3)     # as the pool lies
                s = _pow2_over(x.abs().amax(dim=(2, 3)))
                was = out[w + "_scales"][ids]
                if lead:
                    s[0] = torch.maximum(s[0], was[0])
                y = _round_e4m3(x / s[:, :, None, None])
                kept = out[w + "_pages"][ids]
                if lead:
                    y[0, :, :lead] = _round_e4m3(kept[0, :, :lead] * (was[0] / s[0])[:, None, None])
                tail = lead + n[b] - (count - 1) * page                  # tokens of the last block that hold something now
                y[-1, :, tail:] = kept[-1, :, tail:]
                out[w + "_pages"][ids] = y
                out[w + "_scales"][ids] = s
        return out
    out = torch.zeros((B, M, Hq, dh), dtype=torch.float64, device="cuda")
    group = Hq // Hkv
    for b in range(B):
        if n[b] == 0:
            continue
        T = L[b] + n[b]
        k, v = tokens("k", b, T), tokens("v", b, T)
        unseen = torch.arange(T, device="cuda")[None] > L[b] + torch.arange(n[b], device="cuda")[:, None]
        for h in range(Hq):
            s = rows[b, :n[b], h] @ k[:, h // group].T * dh ** -0.5
            out[b, :n[b], h] = torch.softmax(s.masked_fill(unseen, -math.inf), dim=1) @ v[:, h // group]
    return out
