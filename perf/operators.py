"""The operators of a cache held in 8 bits, as cases whose speed and results can be measured:
writing new tokens into it, the landmark rows of the chunks they complete, decode over it, and
eviction from it by accumulated attention weight.

``own`` says which form ``run`` takes: the plain one (elementary torch operations in float32) or
the calls that a user makes of ``paper_2607_02980_amd.hils``.  ``listed()`` names the cases,
``draw(rng)`` gives more of the same ranges, ``prepare`` makes a case's inputs on the GPU,
``exact`` is the same result in 64 bits and ``work`` what a pass cannot do without.

The cache: a page holds one chunk (64 tokens) of one sequence for every KV head, in e4m3;
a stored x of K (or V) stands for x * kv_scale[page, head, 0 (or 1)], a stored landmark x for
x * kv_scale[page, head, 0].
  k_pages [P, Hkv, 64, d], v_pages [P, Hkv, d, 64], kv_scale [P, Hkv, 2] float32,
  lmk_pages [P, Hl, d], bias_pages [P, Hl] float32, block_table [B, L / 64] int32
"""
import math

import torch

own = False

CHUNK = 64
F8 = torch.float8_e4m3fn
E_MIN = -100  # least exponent of a scale


# ---- the cases -------------------------------------------------------------------------


def _case(name, op, **kw):
    c = dict(op=op, dtype="bf16", B=1, Hq=32, Hkv=8, d=128, N=1, ctx=0, topk=16, window=512, shared_lmk=False,
             bias=False, q_route=False, ragged=False, budget=0, sink=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of a serving batch: every sequence adds one token to a page in use
        _case("append_step_b32", "append", B=32, ctx=131072),
        # a padded batch of prompt pieces of odd lengths that begin and end inside pages, in full precision
        _case("append_ragged_b6_f32", "append", dtype="f32", B=6, Hq=8, Hkv=2, d=64, N=1001, ctx=3333, ragged=True),
        # a long prompt written at once
        _case("append_prompt_64k", "append", N=65536),
        # a decode step in which half of the batch completes a chunk, one landmark query per head
        _case("landmark_step_b48", "landmark", B=48, ctx=32000, shared_lmk=True, ragged=True),
        # the chunks of a 32K prompt
        _case("landmark_prompt_32k", "landmark", N=32768),
        # one interactive chat: the smallest decode step
        _case("decode_4k_b1", "decode", ctx=4095),
        # a small full-precision model: wide groups, landmarks shared by a group, biases, routing queries
        _case("decode_ragged_b5_f32", "decode", dtype="f32", B=5, Hq=16, Hkv=2, d=64, ctx=5000, topk=8, window=256,
              shared_lmk=True, bias=True, q_route=True, ragged=True),
        # drafted tokens verified together
        _case("decode_64k_b8_4new", "decode", B=8, N=4, ctx=65535),
        # long-context decode: a full batch, and few very long sequences
        _case("decode_131k_b32", "decode", B=32, ctx=131072),
        _case("decode_1m_b4", "decode", B=4, ctx=1048576, topk=32),
        # after a decode step: the weights added up, no sequence over its budget
        _case("evict_count_b32", "evict", B=32, ctx=60000, budget=1024, sink=1),
        # very long sequences cut to a quarter of their chunks
        _case("evict_1m_b4", "evict", B=4, ctx=1048576, topk=32, budget=4096, sink=4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "landmark", "decode", "decode", "decode", "evict"])
    hkv, g = rng.choice([(8, 4), (8, 4), (8, 1), (8, 2), (4, 8), (4, 4), (2, 4), (1, 4)])
    c = _case(None, op, Hkv=hkv, Hq=hkv * g, d=rng.choice([64, 128, 128]), topk=rng.choice([4, 8, 16, 16, 32]),
              window=rng.choice([64, 256, 512, 512, 1024]), dtype=rng.choice(["bf16", "bf16", "f32"]))
    if op == "append":
        if rng.random() < 0.5:  # decode steps, drafted tokens
            c.update(B=_log_int(rng, 1, 48), N=rng.choice([1, 1, 2, 5]), ctx=_log_int(rng, 1, 60000))
        else:
            b = _log_int(rng, 1, 12)
            c.update(B=b, N=_log_int(rng, 20, 24000 // b), ctx=rng.choice([0, _log_int(rng, 1, 9000)]),
                     ragged=b > 1 and rng.random() < 0.7)
    elif op == "landmark":
        c.update(shared_lmk=rng.random() < 0.5)
        if rng.random() < 0.5:
            c.update(B=_log_int(rng, 2, 48), ctx=CHUNK * _log_int(rng, 4, 500), ragged=True)
        else:
            c.update(N=_log_int(rng, 100, 24000), ctx=rng.choice([0, _log_int(rng, 1, 9000)]))
    elif op == "decode":
        b = _log_int(rng, 1, 40)
        c.update(B=b, N=rng.choice([1, 1, 1, 2, 4]), ctx=_log_int(rng, 1, min(262144, 4000000 // b)),
                 ragged=b > 1 and rng.random() < 0.5, shared_lmk=g > 1 and rng.random() < 0.3,
                 bias=rng.random() < 0.4, q_route=rng.random() < 0.3)
    else:
        b = _log_int(rng, 1, 48)
        ctx = _log_int(rng, 700, min(1000000, 4000000 // b))
        c.update(B=b, N=rng.choice([1, 1, 1, 4]), ctx=ctx, ragged=b > 1 and rng.random() < 0.5,
                 budget=_log_int(rng, 4, max(8, ctx // 40)), sink=rng.choice([0, 1, 4]))
    return c


# ---- sizes that the case alone determines ------------------------------------------------


def _lens(c):
    """(tokens of each sequence with the new ones, new tokens of each sequence)."""
    B, N, ctx = c["B"], c["N"], c["ctx"]
    if c["op"] == "landmark" and c["ragged"]:  # every other sequence completes a chunk with this token
        return [max(CHUNK, (ctx // CHUNK - 3 * b) * CHUNK) + (b % 2) * (b + 1) % CHUNK for b in range(B)], [1] * B
    new = [N] * B
    if c["op"] == "append" and c["ragged"]:
        new = [max(1, N - b * (N // B) - 3 * b) for b in range(B)]
    if c["ragged"]:
        lo = min(1000, ctx) or 1
        old = [int(lo * (max(ctx, 1) / lo) ** ((b + 0.5) / B)) for b in range(B)]
    else:
        old = [ctx] * B
    return [o + n for o, n in zip(old, new)], new


def _cap(c):
    return (max(_lens(c)[0]) + CHUNK - 1) // CHUNK


def _pieces(c):
    """Window pieces of a row, at most: the chunks that a window of W tokens ending anywhere reaches into."""
    return (c["window"] + 62) // 64 + 1


def _scale(c):
    # with biases 1/8, so that the candidates' scores are exact in 32 bits (see prepare)
    return 0.125 if c["bias"] else float(torch.tensor(c["d"] ** -0.5, dtype=torch.float32))


def _hl(c):
    return c["Hkv"] if c["shared_lmk"] and c["op"] == "decode" else c["Hq"]


def work(case):
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    lens, new = _lens(c)
    Hkv, Hq, d, N, K, W, Hl = c["Hkv"], c["Hq"], c["d"], c["N"], c["topk"], c["window"], _hl(c)
    if c["op"] == "append":
        t = sum(new)
        return {"bytes": 2 * t * Hkv * d * (es + 1) + 8 * Hkv * sum((n + 63) // 64 for n in new), "flops": 4 * t * Hkv * d}
    if c["op"] == "landmark":
        n = sum(a // CHUNK - (a - m) // CHUNK for a, m in zip(lens, new))
        lq = Hq * d * es * (1 if c["shared_lmk"] else n)
        return {"bytes": n * (Hkv * (CHUNK * d + 4) + Hq * (d + 4)) + lq, "flops": 4 * n * Hq * CHUNK * d}
    if c["op"] == "decode":
        nbytes = flops = 0
        for a in lens:
            first, last = a - N, a - 1
            cand = [max(0, i - W + 1) // CHUNK for i in range(first, last + 1)]
            chunks = min(sum(min(K, m) for m in cand), cand[-1]) + last // CHUNK + 1 - cand[0]
            parts = sum(min(K, m) + i // CHUNK + 1 - m for m, i in zip(cand, range(first, last + 1)))
            nbytes += cand[-1] * (Hl * (d + (4 if c["bias"] else 0)) + 4 * Hkv)
            nbytes += chunks * Hkv * (2 * CHUNK * d + 8)
            nbytes += N * Hq * (d * es * (3 if c["q_route"] else 2) + 4) + N * Hkv * 4 * (2 * K + _pieces(c))
            flops += sum(cand) * Hq * 2 * d + parts * Hq * 4 * CHUNK * d
        return {"bytes": nbytes, "flops": flops}
    chunks = sum((a + 63) // 64 for a in lens)
    return {"bytes": 16 * chunks + c["B"] * Hkv * N * 4 * (2 * K + _pieces(c)), "flops": c["B"] * Hkv * N * (K + _pieces(c)) + chunks}


# ---- inputs --------------------------------------------------------------------------------


def _pow2(e, dtype=torch.float32):
    """2^e of whole numbers e, put together from its bits."""
    bits, shift, bias = (torch.int32, 23, 127) if dtype == torch.float32 else (torch.int64, 52, 1023)
    return ((e.to(bits) + bias) << shift).view(dtype)


def _bytes_of(shape, gen, std=64.0):
    """e4m3 values of N(0, std^2), made a slab at a time."""
    n = math.prod(shape)
    x = torch.empty(n, dtype=torch.uint8, device="cuda")
    for i in range(0, n, 1 << 28):
        m = min(1 << 28, n - i)
        y = torch.empty(m, device="cuda").normal_(generator=gen).mul_(std).clamp_(-448, 448)
        x[i:i + m] = y.to(F8).view(torch.uint8)
    return x.view(shape).view(F8)


def _grid(shape, gen, step, most, dtype=torch.float32):
    """Multiples of `step` up to most * step, near N(0, 1): products and sums of such values are exact in 32 bits,
    so the candidates' order, ties included, does not depend on the order of a sum."""
    x = torch.empty(shape, device="cuda").normal_(generator=gen)
    return (x / step).round_().clamp_(-most, most).mul_(step).to(dtype)


def _table(c, lens, gen):
    """Each sequence's pages anywhere among as many as the batch uses and some free ones; -1 past its length."""
    used = [(a + CHUNK - 1) // CHUNK for a in lens]
    P = sum(used) + 8
    perm = torch.randperm(P, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((c["B"], _cap(c)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = perm[at:at + u]
        at += u
    return table, P


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    B, Hq, Hkv, d, N, Hl = c["B"], c["Hq"], c["Hkv"], c["d"], c["N"], _hl(c)
    lens, new = _lens(c)

    def normal(*shape, dtype=dt):
        return torch.empty(shape, device="cuda").normal_(generator=gen).to(dtype)

    t = {"c": c, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"),
         "new": torch.tensor(new, dtype=torch.int32, device="cuda")}
    t["table"], P = _table(c, lens, gen)
    if c["op"] == "evict":
        K, pieces = c["topk"], _pieces(c)
        # what earlier steps left, and one step's weights, on grids whose sums are exact in 32 bits
        t["acc"] = torch.rand((B, _cap(c)), generator=gen, device="cuda").mul_(65536).round_().div_(4096)
        w = torch.rand((B, Hkv, N, K + pieces), generator=gen, device="cuda").mul_(8192).round_().div_(4096 * 64)
        pos = t["lens"].view(B, 1, 1) - N + torch.arange(N, device="cuda")
        cand = (pos - c["window"] + 1).clamp(min=0) // CHUNK  # [B, 1, N]
        pick = torch.rand((B, Hkv, N, K), generator=gen, device="cuda").mul_(cand[..., None].clamp(min=1)).long()
        pick = pick.sort(-1).values
        dup = torch.cat([torch.zeros_like(pick[..., :1], dtype=torch.bool), pick[..., 1:] == pick[..., :-1]], -1)
        pick = torch.where(dup | (cand[..., None] == 0), _cap(c), pick).sort(-1).values
        t["idx"] = torch.where(pick < _cap(c), pick, -1).to(torch.int32)
        piece = cand[..., None] + torch.arange(pieces, device="cuda")
        used = torch.cat([t["idx"] >= 0, (piece <= pos[..., None] // CHUNK).expand(-1, Hkv, -1, -1)], -1)
        t["weights"] = torch.where(used, w, 0.0)
        t["most"] = _cap(c)
        t["acc2"], t["table2"], t["lens2"] = torch.empty_like(t["acc"]), torch.empty_like(t["table"]), torch.empty_like(t["lens"])
        t["freed"] = torch.empty((B, t["most"]), dtype=torch.int32, device="cuda")
        t["nfreed"] = torch.empty(B, dtype=torch.int32, device="cuda")
    else:
        # scales differ from page to page, as the values' ranges do
        e = torch.randint(-7, -4, (P, Hkv, 2), generator=gen, device="cuda")
        t["kv_scale"] = _pow2(e)
        t["k_pages"] = _bytes_of((P, Hkv, CHUNK, d), gen)
        if c["op"] != "landmark":
            t["v_pages"] = _bytes_of((P, Hkv, d, CHUNK), gen)
        if c["op"] != "append":
            t["lmk_pages"] = (_grid((P, Hl, d), gen, 0.25, 15) * 32).to(F8)
            t["bias_pages"] = (_grid((P, Hl), gen, 1 / 1024, 4096) if c["bias"] else
                               torch.zeros((P, Hl), device="cuda"))
        if c["op"] == "append":
            # heads of unlike ranges, so that some pages in use have to change their scale
            r = torch.exp2(torch.empty((B, Hkv, 1, 1), device="cuda").uniform_(-2, 2, generator=gen))
            t["k_new"] = (normal(B, Hkv, N, d, dtype=torch.float32) * r).to(dt)
            t["v_new"] = (normal(B, Hkv, N, d, dtype=torch.float32) * r).to(dt)
        elif c["op"] == "landmark":
            t["lq"] = normal(Hl, d) if c["shared_lmk"] else normal(B, Hl, (N + CHUNK - 1) // CHUNK, d)
        else:
            exact_q = _grid((B, Hq, N, d), gen, 1 / 16, 64, dt)
            t["q_route"] = exact_q if c["q_route"] else None
            t["q"] = normal(B, Hq, N, d) if c["q_route"] else exact_q
    if own:
        from paper_2607_02980_amd import hils

        flags = hils.HILS_FLAG_SHARED_LMK_QUERY if c["op"] == "landmark" and c["shared_lmk"] else 0
        t["p"] = hils.Params(B=B, Hq=Hq, Hkv=Hkv, N=N, L=_cap(c) * CHUNK, d=d, chunk=CHUNK, topk=c["topk"],
                             window=c["window"], scale=_scale(c), dtype=c["dtype"], Hl=Hl, flags=flags)
        if c["op"] == "decode":  # a decode loop keeps its outputs and its workspace
            p, f32 = t["p"], torch.float32
            t["out"] = torch.empty((B, Hq, N, d), dtype=dt, device="cuda")
            t["lse"] = torch.empty((B, Hq, N), dtype=f32, device="cuda")
            t["idx"] = torch.empty((B, Hkv, N, c["topk"]), dtype=torch.int32, device="cuda")
            t["weights"] = torch.empty((B, Hkv, N, c["topk"] + _pieces(c)), dtype=f32, device="cuda")
            t["ws"] = torch.empty(max(1, hils.hils_workspace_size(p, hils.HILS_OP_DECODE_Q8)), dtype=torch.uint8, device="cuda")
    return t


# ---- one pass --------------------------------------------------------------------------------


def run(state):
    t = state
    op = t["c"]["op"]
    if own:
        from paper_2607_02980_amd import hils

        if op == "append":
            hils.hils_q8_append(t["p"], t["k_new"], t["v_new"], t["k_pages"], t["v_pages"], t["kv_scale"], t["table"],
                                seqlens=t["lens"], newlens=t["new"])
            return {"k_pages": t["k_pages"], "v_pages": t["v_pages"], "kv_scale": t["kv_scale"]}
        if op == "landmark":
            hils.hils_q8_landmark_fwd(t["p"], t["lq"], t["k_pages"], t["kv_scale"], t["table"], t["lmk_pages"],
                                      t["bias_pages"], seqlens=t["lens"], newlens=t["new"])
            return {"lmk_pages": t["lmk_pages"], "bias_pages": t["bias_pages"]}
        if op == "decode":
            out, lse, idx, weights = hils.hils_decode_q8_fwd(
                t["p"], t["q"], t["k_pages"], t["v_pages"], t["kv_scale"], t["lmk_pages"], t["table"],
                bias_pages=t["bias_pages"] if t["c"]["bias"] else None, q_route=t["q_route"], seqlens=t["lens"], out=t["out"],
                lse=t["lse"], idx=t["idx"], weights=t["weights"], workspace=t["ws"])
            return {"out": out, "lse": lse, "idx": idx, "weights": weights}
        acc, table, lens, freed, nfreed = hils.hils_cache_evict(
            t["p"], t["acc"], t["table"], t["lens"], budget=t["c"]["budget"], sink=t["c"]["sink"], max_evict=t["most"],
            weights=t["weights"], idx=t["idx"], acc_out=t["acc2"], table_out=t["table2"], seqlens_out=t["lens2"],
            freed=t["freed"], nfreed=t["nfreed"])
        return {"acc": acc, "block_table": table, "seqlens": lens, "freed": freed, "nfreed": nfreed}
    return {"append": _plain_append, "landmark": _plain_landmark, "decode": _plain_decode, "evict": _plain_evict}[op](t)


def _take(pool, pages, heads=None):
    """Values of e4m3 pages in float32, without their scales."""
    raw = pool.view(torch.uint8)
    return (raw[pages] if heads is None else raw[pages, heads]).view(F8).float()


def _plain_append(t):
    c = t["c"]
    B, Hkv, d, N = c["B"], c["Hkv"], c["d"], c["N"]
    dev = t["k_new"].device
    start = (t["lens"] - t["new"]).long()
    most = (N + 62) // CHUNK + 1  # chunks that N tokens reach into
    chunk = start[:, None] // CHUNK + torch.arange(most, device=dev)  # [B, most]
    row = chunk[..., None] * CHUNK + torch.arange(CHUNK, device=dev)  # positions [B, most, 64]
    n = row - start[:, None, None]
    is_new = (n >= 0) & (n < t["new"][:, None, None])
    is_old = n < 0
    hit = is_new.any(-1)  # chunks that get a token
    at = torch.nonzero(hit)
    b = at[:, 0]
    page = t["table"][b, chunk[hit]].long()
    is_new, is_old, n = is_new[hit][:, None, :, None], is_old[hit][:, None, :, None], n[hit]  # [m, 1, 64, 1]
    had = is_old.any(2)  # [m, 1, 1]: the chunk holds older tokens
    for which, x, pool in ((0, t["k_new"], t["k_pages"]), (1, t["v_new"], t["v_pages"])):
        rows = x.transpose(1, 2)[b[:, None], n.clamp(0, N - 1)].transpose(1, 2).float()  # [m, Hkv, 64, d]
        amax = torch.where(is_new & rows.isfinite(), rows.abs(), 0.0).amax((2, 3))  # [m, Hkv]
        frac, ex = torch.frexp(amax)
        e = torch.where(amax > 0, torch.where(frac <= 0.875, ex - 9, ex - 8), E_MIN).clamp(min=E_MIN)
        need = _pow2(e)
        old = t["kv_scale"][page, :, which]
        s = torch.where(had[..., 0], torch.maximum(old, need), need)
        held = pool.view(torch.uint8)[page]  # K [m, Hkv, 64, d], V [m, Hkv, d, 64]
        held = held.transpose(2, 3) if which else held
        moved = (held.contiguous().view(F8).float() * (old / s)[..., None, None]).to(F8).view(torch.uint8)
        fresh = torch.where(rows.isfinite(), rows / s[..., None, None], float("nan")).to(F8).view(torch.uint8)
        got = torch.where(is_new, fresh, torch.where(is_old, moved, held))
        pool.view(torch.uint8)[page] = got.transpose(2, 3).contiguous() if which else got
        t["kv_scale"][page, :, which] = s
    return {"k_pages": t["k_pages"], "v_pages": t["v_pages"], "kv_scale": t["kv_scale"]}


def _plain_landmark(t):
    c = t["c"]
    G, dev = c["Hq"] // c["Hkv"], t["k_pages"].device
    first = (t["lens"] - t["new"]).long() // CHUNK  # the first chunk that may become complete
    most = (c["N"] + CHUNK - 1) // CHUNK
    chunk = first[:, None] + torch.arange(most, device=dev)
    at = torch.nonzero(chunk < t["lens"][:, None] // CHUNK)
    page = t["table"][at[:, 0], chunk[at[:, 0], at[:, 1]]].long()
    k = _take(t["k_pages"], page).repeat_interleave(G, 1)  # [m, Hl, 64, d], in units of its scale
    ks = t["kv_scale"][page, :, 0].repeat_interleave(G, 1)
    lq = t["lq"].float() if c["shared_lmk"] else t["lq"].transpose(1, 2)[at[:, 0], at[:, 1]].float()
    s = _scale(c) * ks[..., None] * (k * lq[..., None, :]).sum(-1)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    t["lmk_pages"].view(torch.uint8)[page] = (p[..., None] * k).sum(-2).to(F8).view(torch.uint8)
    t["bias_pages"][page] = torch.where(p > 0, -p * torch.log(p), 0.0).sum(-1)
    return {"lmk_pages": t["lmk_pages"], "bias_pages": t["bias_pages"]}


def _plain_decode(t):
    c = t["c"]
    B, Hq, Hkv, N, d, K, W = c["B"], c["Hq"], c["Hkv"], c["N"], c["d"], c["topk"], c["window"]
    G, nC, Hl, scale, dev = Hq // Hkv, t["table"].shape[1], _hl(c), _scale(c), t["q"].device
    inf = float("inf")
    page = t["table"].long().clamp(min=0)
    i = t["lens"].long()[:, None] - N + torch.arange(N, device=dev)  # [B, N]
    cand = (i - W + 1).clamp(min=0) // CHUNK
    # every candidate's score for every head
    lm = _take(t["lmk_pages"], page) * t["kv_scale"][page, :, 0].repeat_interleave(Hl // Hkv, 2)[..., None]
    lm = lm.transpose(1, 2).repeat_interleave(Hq // Hl, 1)  # [B, Hq, nC, d]
    qr = (t["q_route"] if c["q_route"] else t["q"]).float()
    s = scale * torch.matmul(lm, qr.transpose(2, 3).contiguous())  # [B, Hq, nC, N]
    if c["bias"]:
        s = s + t["bias_pages"][page].transpose(1, 2).repeat_interleave(Hq // Hl, 1)[..., None]
    s = s.transpose(2, 3).reshape(B, Hkv, G, N, nC)
    # the K best of a group, by the best of its heads; ties to the lower index
    open_ = (torch.arange(nC, device=dev) < cand[..., None])[:, None].expand(B, Hkv, N, nC)
    best = torch.sort(s.amax(2).masked_fill(~open_, -inf), dim=-1, descending=True, stable=True).indices[..., :K]
    idx = torch.where(open_.gather(-1, best), best, nC).sort(-1).values
    idx = torch.nn.functional.pad(idx, (0, K - idx.shape[-1]), value=nC)
    chosen = idx < nC
    # the parts of a row: its chosen chunks, then the pieces of its window
    piece = cand[..., None] + torch.arange(_pieces(c), device=dev)  # [B, N, pieces]
    seen = (i[..., None] - piece * CHUNK + 1).clamp(0, CHUNK)[:, None].expand(-1, Hkv, -1, -1)
    ids = torch.cat([torch.where(chosen, idx, 0), piece.clamp(max=nC - 1)[:, None].expand(-1, Hkv, -1, -1)], -1)
    nk = torch.cat([chosen.long() * CHUNK, seen], -1)  # keys of each part [B, Hkv, N, P]
    pg = page[:, None, None].expand(B, Hkv, N, nC).gather(-1, ids)
    head = torch.arange(Hkv, device=dev).view(1, Hkv, 1, 1)
    kvs = t["kv_scale"][pg, head]
    in_part = torch.arange(CHUNK, device=dev) < nk[..., None]  # [B, Hkv, N, P, 64]
    k = torch.where(in_part[..., None], _take(t["k_pages"], pg, head), 0.0) * kvs[..., 0, None, None]
    v = torch.where(in_part[..., None, :], _take(t["v_pages"], pg, head), 0.0) * kvs[..., 1, None, None]
    q = t["q"].float().view(B, Hkv, G, N, d).permute(0, 1, 3, 4, 2).unsqueeze(3)  # [B, Hkv, N, 1, d, G]
    x = scale * torch.matmul(k, q.expand(-1, -1, -1, k.shape[3], -1, -1).contiguous())  # [B, Hkv, N, P, 64, G]
    x = x.masked_fill(~in_part[..., None], -inf)
    top = x.amax(-2, keepdim=True)
    e = torch.exp(x - torch.where(top == -inf, 0.0, top))
    l = e.sum(-2)  # [B, Hkv, N, P, G]
    mass = torch.where(l > 0, top.squeeze(-2) + torch.log(l), -inf)
    o = torch.matmul(v, e)  # [B, Hkv, N, P, d, G]
    # the fusion
    z = s.gather(-1, torch.where(chosen, idx, 0)[:, :, None].expand(-1, -1, G, -1, -1)).permute(0, 1, 3, 4, 2)
    z = torch.cat([z.masked_fill(~chosen[..., None], -inf), mass[..., K:, :]], 3)
    lse = torch.logsumexp(z, 3)  # [B, Hkv, N, G]
    w = torch.exp(z - lse.unsqueeze(3))
    out = (torch.where(l > 0, w / l, 0.0).unsqueeze(4) * o).sum(3)  # [B, Hkv, N, d, G]
    return {"out": out.permute(0, 1, 4, 2, 3).reshape(B, Hq, N, d).to(t["q"].dtype),
            "lse": lse.transpose(2, 3).reshape(B, Hq, N), "idx": torch.where(chosen, idx, -1).to(torch.int32),
            "weights": w.sum(-1)}


def _plain_evict(t):
    c = t["c"]
    B, Hkv, N, K, nC, dev = c["B"], c["Hkv"], c["N"], c["topk"], t["acc"].shape[1], t["acc"].device
    i = t["lens"].long()[:, None] - N + torch.arange(N, device=dev)
    cand = (i - c["window"] + 1).clamp(min=0) // CHUNK
    piece = (cand[..., None] + torch.arange(_pieces(c), device=dev))[:, None].expand(-1, Hkv, -1, -1)
    ids = torch.cat([t["idx"].long(), piece], -1).reshape(B, -1)
    ok = (ids >= 0) & (ids < nC)
    acc = t["acc"].scatter_add(1, torch.where(ok, ids, 0), torch.where(ok, t["weights"].reshape(B, -1), 0.0))
    last = cand[:, -1]
    c_of = torch.arange(nC, device=dev)
    free = (c_of >= c["sink"]) & (c_of < last[:, None])
    n = torch.minimum((last - c["budget"]).clamp(min=0), free.sum(1)).clamp(max=t["most"])
    order = torch.sort(torch.where(free, acc, float("inf")), dim=1, stable=True).indices
    rank = torch.empty_like(order).scatter_(1, order, c_of.expand(B, -1))
    gone = free & (rank < n[:, None])
    kept = torch.sort(gone.to(torch.uint8), dim=1, stable=True).indices  # the kept chunks in order, then the others
    tail = c_of >= (nC - n)[:, None]
    listed_ = torch.sort((~gone).to(torch.uint8), dim=1, stable=True).indices[:, :t["most"]]
    return {"acc": torch.where(tail, 0.0, acc.gather(1, kept)),
            "block_table": torch.where(tail, -1, t["table"].gather(1, kept)),
            "seqlens": (t["lens"] - CHUNK * n).to(torch.int32),
            "freed": torch.where(c_of[:t["most"]] < n[:, None], t["table"].gather(1, listed_), -1),
            "nfreed": n.to(torch.int32)}


# ---- the same in 64 bits, one sequence at a time -----------------------------------------------


def _round8(x):
    """Nearest e4m3 value (ties to even) of float64 values within +-448."""
    a = x.abs()
    ex = torch.frexp(a)[1] - 1
    step = _pow2(ex.clamp(min=-6) - 3, torch.float64)
    return torch.sign(x) * torch.round(a / step) * step


def _exact_append(c, t):
    k, v, sc = (t[n].double() for n in ("k_pages", "v_pages", "kv_scale"))
    lens, new = _lens(c)
    for b in range(c["B"]):
        start = lens[b] - new[b]
        for ch in range(start // CHUNK, (lens[b] - 1) // CHUNK + 1):
            lo, hi = max(start, ch * CHUNK), min(lens[b], (ch + 1) * CHUNK)
            r0, r1, page = lo - ch * CHUNK, hi - ch * CHUNK, int(t["table"][b, ch])
            for which, x, pool in ((0, t["k_new"], k), (1, t["v_new"], v.transpose(2, 3))):
                y = x[b, :, lo - start:hi - start].double()
                amax = y.abs().amax((1, 2))
                s = _pow2(torch.ceil(torch.log2(amax / 448)).clamp(min=E_MIN), torch.float64)
                if r0 > 0:
                    s = torch.maximum(s, sc[page, :, which])
                    pool[page, :, :r0] = _round8(pool[page, :, :r0] * (sc[page, :, which] / s)[:, None, None])
                pool[page, :, r0:r1] = _round8(y / s[:, None, None])
                sc[page, :, which] = s
    return {"k_pages": k, "v_pages": v, "kv_scale": sc}


def _exact_landmark(c, t):
    lm, bias = t["lmk_pages"].double(), t["bias_pages"].double()
    lens, new = _lens(c)
    G = c["Hq"] // c["Hkv"]
    for b in range(c["B"]):
        first, end = (lens[b] - new[b]) // CHUNK, lens[b] // CHUNK
        for j0 in range(first, end, 64):
            page = t["table"][b, j0:min(end, j0 + 64)].long()
            k = _take(t["k_pages"], page).double()  # [m, Hkv, 64, d]
            lq = t["lq"].double()
            lq = lq[None] if c["shared_lmk"] else lq[b, :, j0 - first:j0 - first + len(page)].transpose(0, 1)
            lq = lq.expand(len(page), -1, -1).reshape(len(page), c["Hkv"], G, c["d"])
            s = _scale(c) * t["kv_scale"][page, :, 0].double()[..., None, None] * torch.matmul(lq, k.transpose(2, 3).contiguous())
            logp = torch.log_softmax(s, -1)
            p = logp.exp()
            lm[page] = torch.matmul(p, k).reshape(len(page), c["Hq"], c["d"])
            bias[page] = -(p * logp).sum(-1).reshape(len(page), c["Hq"])
    return {"lmk_pages": lm, "bias_pages": bias}


def _exact_decode(c, t):
    f64, dev = torch.float64, "cuda"
    B, Hq, Hkv, N, d, K, W = c["B"], c["Hq"], c["Hkv"], c["N"], c["d"], c["topk"], c["window"]
    G, Hl, scale, P = Hq // Hkv, _hl(c), _scale(c), K + _pieces(c)
    r = {"out": torch.zeros(B, Hq, N, d, dtype=f64, device=dev), "lse": torch.zeros(B, Hq, N, dtype=f64, device=dev),
         "idx": torch.full((B, Hkv, N, K), -1, dtype=torch.int32, device=dev),
         "weights": torch.zeros(B, Hkv, N, P, dtype=f64, device=dev)}
    heads = torch.arange(Hkv, device=dev)[:, None]
    for b, length in enumerate(_lens(c)[0]):
        table = t["table"][b].long()
        for n in range(N):
            i = length - N + n
            nc = max(0, i - W + 1) // CHUNK
            q = t["q"][b, :, n].to(f64).view(Hkv, G, d)

            def attend(ids):  # ids [Hkv, m]: logits [Hkv, m, 64, G], values [Hkv, m, 64, d]
                pg = table[ids]
                sc = t["kv_scale"][pg, heads].to(f64)
                k = _take(t["k_pages"], pg, heads).to(f64) * sc[..., 0, None, None]
                v = _take(t["v_pages"], pg, heads).to(f64) * sc[..., 1, None, None]
                return scale * torch.matmul(k, q.transpose(1, 2).contiguous()[:, None]), v.transpose(2, 3).contiguous()

            own_ids = torch.arange(nc, i // CHUNK + 1, device=dev).expand(Hkv, -1)
            x, v = attend(own_ids)
            ahead = own_ids[..., None] * CHUNK + torch.arange(CHUNK, device=dev) > i
            x = x.masked_fill(ahead[..., None], -math.inf)
            z, cat = [torch.logsumexp(x, 2)], [(x, v)]
            if nc:
                qr = t["q_route"][b, :, n].to(f64).view(Hkv, G, d) if c["q_route"] else q
                pg = table[:nc]
                lm = _take(t["lmk_pages"], pg).to(f64).view(nc, Hkv, Hl // Hkv, d)
                lm = lm * t["kv_scale"][pg, :, 0].to(f64)[..., None, None]
                s = scale * (lm * qr).sum(-1) if Hl == Hq else scale * torch.matmul(lm, qr.transpose(1, 2).contiguous())[:, :, 0]
                s = s + t["bias_pages"][pg].to(f64).view(nc, Hkv, Hl // Hkv) if c["bias"] else s  # [nc, Hkv, G]
                sig = s.amax(-1).T.contiguous()
                m = min(K, nc)
                idx = torch.sort(sig, dim=-1, descending=True, stable=True).indices[:, :m].sort(-1).values
                r["idx"][b, :, n, :m] = idx.to(torch.int32)
                z.insert(0, s.transpose(0, 1).gather(1, idx[..., None].expand(-1, -1, G)))
                cat.insert(0, attend(idx))
            lse = torch.logsumexp(torch.cat(z, 1), 1)  # [Hkv, G]
            o = 0
            for (x, v), logit in zip(cat, z):
                w = torch.exp(logit - lse[:, None])  # [Hkv, m, G]
                o = o + torch.matmul((torch.softmax(x, 2) * w[:, :, None]).flatten(1, 2).transpose(1, 2).contiguous(), v.flatten(1, 2))
            r["out"][b, :, n], r["lse"][b, :, n] = o.reshape(Hq, d), lse.reshape(-1)
            if nc:
                r["weights"][b, :, n, :z[0].shape[1]] = torch.exp(z[0] - lse[:, None]).sum(-1)
            r["weights"][b, :, n, K:K + z[-1].shape[1]] = torch.exp(z[-1] - lse[:, None]).sum(-1)
    return r


def _exact_evict(c, t):
    K, N, W, nC = c["topk"], c["N"], c["window"], t["acc"].shape[1]
    acc, table, idx, wt = (t[n].cpu() for n in ("acc", "table", "idx", "weights"))
    acc, lens = acc.double(), _lens(c)[0]
    freed, counts, ends = torch.full((c["B"], t["most"]), -1, dtype=torch.int32), [], []
    for b in range(c["B"]):
        for n in range(N):
            i = lens[b] - N + n
            nc = max(0, i - W + 1) // CHUNK
            for g in range(c["Hkv"]):
                sel = idx[b, g, n][idx[b, g, n] >= 0].long()
                acc[b, sel] += wt[b, g, n, :len(sel)].double()
                m = i // CHUNK + 1 - nc
                acc[b, nc:nc + m] += wt[b, g, n, K:K + m].double()
        able = list(range(c["sink"], nc))
        count = min(max(0, nc - c["budget"]), len(able), t["most"])
        total = acc[b].tolist()
        gone = sorted(sorted(able, key=lambda ch: (total[ch], ch))[:count])
        out = set(gone)
        kept = [ch for ch in range(nC) if ch not in out]
        freed[b, :count] = table[b, gone]
        acc[b] = torch.cat([acc[b, kept], torch.zeros(count, dtype=torch.float64)])
        table[b] = torch.cat([table[b, kept], torch.full((count,), -1, dtype=torch.int32)])
        counts.append(count)
        ends.append(lens[b] - CHUNK * count)
    return {"acc": acc, "block_table": table, "seqlens": torch.tensor(ends, dtype=torch.int32), "freed": freed,
            "nfreed": torch.tensor(counts, dtype=torch.int32)}


def exact(case, seed):
    t = prepare(case, seed)
    return {"append": _exact_append, "landmark": _exact_landmark, "decode": _exact_decode, "evict": _exact_evict}[case["op"]](case, t)
