"""Chunks of new tokens on the compressed cache, as cases that can be timed and checked.

Each case is one pass through the public entry points of `paper_2601_18383_amd.binding`, as a program calls them, or
(`own` false) through the same mathematics in elementary torch operations, 32 bits throughout and rounded once:

  rotate    rotary positions of a chunk's queries and keys, one to four axes; `inverse` is the gradient of it
  prompt    a prompt fills an empty cache: its rows are appended and attended, question slots throughout
  attend    the last tokens of every sequence attend to the cache, each to what lies before it and to itself
  score     the same, and the attention weight that every cached slot receives from them
  shaped    the same as attend, with a cap on the logits, a bias by distance, a window, documents or a prefix

Shapes are those of configs.py (model geometry, budgets, batch sizes) and of the tests, the rest is generic; `draw`
spreads sizes over the ranges these stand for.  Queries lie around a mean direction, a few keys in it are critical.
Cached positions have the gaps that evictions leave, other gaps in every KV head.
"""
import math

import torch

own = False
DEV = "cuda"
PAGE = 64
NEVER = -(1 << 30)


# ---- the cases ---------------------------------------------------------------------------------------------------

def _rotate(name, batch, tokens, hq, hkv, d, pairs, axes, adjacent, inverse, far):
    c = dict(kind="rotate", batch=batch, tokens=tokens, hq=hq, hkv=hkv, d=d, pairs=pairs, axes=axes, adjacent=adjacent,
             inverse=inverse, far=far)
    return dict(c, name=name) if name else c


def _chunk(name, kind, batch, hq, hkv, d, cached, tokens, ragged=False, paged=False, cap=0.0, slopes=False, window=0,
           documents=0, prefix=0, gaps=0):
    """cached: slots before the chunk; ragged: lengths of both differ between sequences; gaps: positions evicted."""
    c = dict(kind=kind, batch=batch, hq=hq, hkv=hkv, d=d, cached=cached, tokens=tokens, ragged=ragged, paged=paged,
             cap=cap, slopes=slopes, window=window, documents=documents, prefix=prefix, gaps=gaps)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of each of 32 sequences (cfg3's batch and heads) far into its answer: latency counts
        _rotate("rotate_token_b32_qwen", 32, 1, 28, 4, 128, 64, 1, False, False, 32768),
        # a prompt of images on the 8B-shaped heads: time, height and width
        _rotate("rotate_image_prompt_llama", 4, 2048, 32, 8, 128, 64, 3, False, False, 4096),
        # the gradient on the small heads of cfg1: part of the head turned, neighbours paired, an odd length
        _rotate("rotate_gradient_small", 2, 999, 8, 2, 64, 24, 2, True, True, 100000),
        # the prompts of a batch of 64 (cfg4) into an empty cache
        _chunk("prompt_b64_llama", "prompt", 64, 32, 8, 128, 0, 512),
        # four drafted tokens of every sequence of the headline workload (cfg3), on pages
        _chunk("attend_draft_b32_qwen_paged", "attend", 32, 28, 4, 128, 2464, 4, paged=True, gaps=9000),
        # one user's long document, a chunk of it on top of what was read before
        _chunk("attend_long_b1_llama", "attend", 1, 32, 8, 128, 16384, 2048),
        # a padded batch of short odd chunks on small heads (cfg1's), some of them empty, on pages
        _chunk("attend_ragged_small_paged", "attend", 5, 8, 2, 64, 333, 77, ragged=True, paged=True, gaps=500),
        # a known answer of 512 tokens (teacher forcing) on the headline workload, and whom it attends to
        _chunk("score_answer_b32_qwen", "score", 32, 28, 4, 128, 2464, 512, gaps=9000),
        # a short tool result for one user (cfg2's cache)
        _chunk("score_short_b1_llama", "score", 1, 32, 8, 128, 4500, 16, gaps=11000),
        # single tokens with capped logits and a window, on the headline workload's cache
        _chunk("shaped_token_b32_qwen", "shaped", 32, 28, 4, 128, 2464, 1, cap=50.0, window=4096, gaps=9000),
        # prompts that open with an image: its tokens see each other both ways; on pages
        _chunk("shaped_prefix_b8_llama_paged", "shaped", 8, 32, 8, 128, 0, 1024, paged=True, prefix=577),
        # documents packed into one long prompt, bias by distance
        _chunk("shaped_documents_b2_llama", "shaped", 2, 32, 8, 128, 0, 4096, slopes=True, documents=9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv, d = rng.choice([(28, 4, 128), (32, 8, 128), (8, 2, 64), (6, 6, 128), (16, 1, 64), (16, 2, 128)])
    if rng.random() < 0.25:
        tokens = _log(rng, 1, 4096)
        batch = min(_log(rng, 1, 128), max(1, 8192 // tokens))
        pairs = rng.choice([d // 2, d // 2, d // 4, 24])
        return _rotate(None, batch, tokens, hq, hkv, d, pairs, rng.randint(1, 4), rng.random() < 0.4,
                       rng.random() < 0.4, _log(rng, 100, 1 << 20))
    kind = rng.choice(["prompt", "attend", "attend", "score", "shaped", "shaped"])
    tokens = _log(rng, 1, 4096) if kind != "prompt" else _log(rng, 16, 4096)
    cached = 0 if kind == "prompt" else _log(rng, 1, 20000)
    # (no more work than the largest listed case: pairs of query and key over batch and heads)
    most = 32 * 28 * 512 * 2464 // 2
    batch = max(1, min(_log(rng, 1, 64), most // (hq * tokens * (cached + tokens)), 32000000 // (hkv * d * (cached + tokens))))
    while hq * tokens * (cached + tokens) > most:
        tokens = (tokens + 1) // 2
    if kind == "prompt":
        return _chunk(None, kind, batch, hq, hkv, d, 0, tokens, ragged=rng.random() < 0.5)
    c = _chunk(None, kind, batch, hq, hkv, d, cached, tokens, ragged=rng.random() < 0.5, paged=rng.random() < 0.5,
               gaps=rng.choice([0, _log(rng, 1, 20000)]))
    if kind == "shaped":
        c["cap"] = rng.choice([0.0, 30.0, 50.0])
        c["slopes"] = rng.random() < 0.5
        c["window"] = rng.choice([0, _log(rng, 16, 8192)])
        c["documents"] = rng.choice([0, 0, rng.randint(2, 12)])
        c["prefix"] = rng.choice([0, 0, rng.randint(1, tokens)])
        if not (c["cap"] or c["slopes"] or c["window"] or c["documents"] or c["prefix"]):
            c["cap"] = 30.0
    return c


# ---- the inputs ----------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rotate_inputs(case, seed):
    g = _gen(seed)
    B, T, d, P, A = case["batch"], case["tokens"], case["d"], case["pairs"], case["axes"]
    x = dict(q=torch.randn((B, T, case["hq"], d), generator=g, device=DEV).to(torch.bfloat16),
             k=torch.randn((B, T, case["hkv"], d), generator=g, device=DEV).to(torch.bfloat16))
    # tokens follow each other on the first axis; the others are places in a grid
    start = torch.randint(0, max(1, case["far"]), (B, 1), generator=g, device=DEV)
    rows = [start + torch.arange(T, device=DEV)[None]]
    for _ in range(A - 1):
        rows.append(torch.randint(0, 1 + case["far"] // 16, (B, T), generator=g, device=DEV))
    x["positions"] = torch.stack(rows).to(torch.int32)
    x["freq"] = (10000.0 ** (-torch.arange(P, device=DEV, dtype=torch.float64) / P)).to(torch.float32)
    x["axis"] = (torch.arange(P, device=DEV) * A // P).to(torch.uint8)
    return x


def _chunk_inputs(case, seed):
    g = _gen(seed)
    B, hq, hkv, d, T, n = case["batch"], case["hq"], case["hkv"], case["d"], case["tokens"], case["cached"]
    x = {}
    x["n_new"] = torch.full((B,), T, dtype=torch.int32, device=DEV)
    x["n_old"] = torch.full((B,), n, dtype=torch.int32, device=DEV)
    if case["ragged"]:
        # the first sequence is as long as they come, the others anything down to nothing new
        r = torch.rand((B,), generator=g, device=DEV)
        x["n_new"] = torch.floor(r * (T + 1)).to(torch.int32).clamp(max=T)
        x["n_new"][0] = T
        r = torch.rand((B,), generator=g, device=DEV)
        x["n_old"] = torch.floor((1 - r * r) * (n + 1)).to(torch.int32).clamp(max=n)
        x["n_old"][0] = n
    rows = n + T                               # logical rows: [0, n_old) cached, then the chunk's n_new
    u = torch.randn((B, 1, hkv, d), generator=g, device=DEV)
    k = torch.randn((B, rows, hkv, d), generator=g, device=DEV)
    critical = torch.rand((B, rows, hkv, 1), generator=g, device=DEV) < 0.02
    k += critical * 0.4 * u
    x["k"] = k.to(torch.bfloat16)
    x["v"] = torch.randn((B, rows, hkv, d), generator=g, device=DEV).to(torch.bfloat16)
    uq = u.repeat_interleave(hq // hkv, dim=2)
    x["q"] = (0.8 * torch.randn((B, T, hq, d), generator=g, device=DEV) + 0.6 * uq).to(torch.bfloat16)
    # positions [B][hkv][rows]: a cached prefix, kept tokens with gaps, the newest without; then the chunk
    j = torch.arange(rows, device=DEV)
    kept = torch.floor(torch.rand((B, hkv, rows), generator=g, device=DEV).sort(dim=-1).values * case["gaps"])
    lead, tail = n // 8, n // 8
    inside = (j >= lead) & (j[None] < (x["n_old"][:, None] - tail))
    ahead = (j < lead) & (j[None] < (x["n_old"][:, None] - tail))
    pos = j + torch.where(inside[:, None], kept, torch.where(ahead[:, None], 0.0, float(case["gaps"])))
    x["pos"] = pos.to(torch.int32)
    x["next"] = x["n_old"] + case["gaps"]      # the position of a chunk's first token
    x["own_pos"] = x["next"][:, None] + torch.arange(T, device=DEV, dtype=torch.int32)
    x["first"] = x["last"] = x["slope"] = None
    if case["kind"] == "shaped":
        end = n + case["gaps"] + T
        if case["documents"]:
            starts = torch.randint(0, end, (B, case["documents"]), generator=g, device=DEV).to(torch.int32)
            starts = torch.where(starts[:, None] <= x["own_pos"][..., None], starts[:, None], 0)
            x["first"] = starts.max(dim=-1).values.to(torch.int32).contiguous()
        if case["prefix"]:
            edge = x["next"][:, None] + (case["prefix"] - 1)
            x["last"] = torch.maximum(x["own_pos"], edge).where(x["own_pos"] <= edge, x["own_pos"]).to(torch.int32).contiguous()
        if case["slopes"]:
            x["slope"] = (2.0 ** (-8.0 * (1 + torch.arange(hq, device=DEV, dtype=torch.float64)) / hq)).to(torch.float32)
    return x


def _dense(x, name, capacity):
    """Logical rows [B][rows][hkv][d] as a cache lies: [B][hkv][capacity][d]."""
    rows = x[name].permute(0, 2, 1, 3)
    out = torch.zeros((rows.shape[0], rows.shape[1], capacity, rows.shape[3]), dtype=torch.bfloat16, device=DEV)
    out[:, :, :rows.shape[2]] = rows
    return out


def _rows_of_chunk(x, name, T):
    """The chunk's own rows [B][T][hkv][d] out of the logical ones (those behind n_new are padding)."""
    at = (x["n_old"].long()[:, None] + torch.arange(T, device=DEV)).clamp(max=x[name].shape[1] - 1)
    return torch.gather(x[name], 1, at[..., None, None].expand(-1, -1, *x[name].shape[2:])).contiguous()


def prepare(case, seed):
    if case["kind"] == "rotate":
        x = _rotate_inputs(case, seed)
        st = dict(case=case, q_out=torch.empty_like(x["q"]), k_out=torch.empty_like(x["k"]), **x)
        if own:
            from paper_2601_18383_amd import binding as B
            st["rotary"] = B.Rotary(case["d"], x["freq"], x["axis"], case["axes"],
                                    B.DYNTS_PAIR_ADJACENT if case["adjacent"] else B.DYNTS_PAIR_HALVES)
        return st
    x = _chunk_inputs(case, seed)
    Nb, hq, hkv, d, T, n = case["batch"], case["hq"], case["hkv"], case["d"], case["tokens"], case["cached"]
    capacity = (n + T + PAGE - 1) // PAGE * PAGE
    st = dict(case=case, q=x["q"], n_new=x["n_new"], n_old=x["n_old"], own_pos=x["own_pos"], pos=x["pos"], slope=x["slope"],
              first=x["first"], last=x["last"], capacity=capacity,
              out=torch.zeros((Nb, T, hq, d), dtype=torch.bfloat16, device=DEV),
              lse=torch.zeros((Nb, T, hq), dtype=torch.float32, device=DEV))
    if case["kind"] == "score":
        st["received"] = torch.zeros((Nb, hkv, capacity), dtype=torch.float32, device=DEV)
    total = (x["n_old"] + x["n_new"]).to(torch.int32)
    if case["kind"] == "prompt":
        st["k_new"], st["v_new"] = _rows_of_chunk(x, "k", T), _rows_of_chunk(x, "v", T)
    K, V = _dense(x, "k", capacity), _dense(x, "v", capacity)
    if own:
        from paper_2601_18383_amd import binding as B
        kw = dict(softmax_scale=0.0, device=DEV + ":0")
        # (the budget does not matter here: nothing is evicted)
        cache = (B.PagedCache if case["paged"] else B.Cache)(1, Nb, hq, hkv, d, capacity, 0, 0, 1, **kw)
        st["cache"] = cache
        st["scratch"] = torch.empty(B.dynts_chunk_scratch_bytes(cache.cfg, T), dtype=torch.uint8, device=DEV)
        if case["kind"] != "prompt":
            B.dynts_prefill(cache.ctx, 0, K, V, total)
            cache.n_prompt.zero_()
            cache.S.zero_()
            cache.pos[0, :, :, :n + T] = x["pos"]
        if case["kind"] == "shaped":
            st["shaping"] = B.Shaping(softcap=case["cap"], window=case["window"], slope=x["slope"], first=x["first"],
                                      last=x["last"])
    elif case["paged"]:
        # pages in no order, as a pool hands them out, and a table of them
        per = capacity // PAGE
        order = torch.randperm(Nb * hkv * per, generator=_gen(seed + 1), device=DEV)
        st["table"] = order.reshape(Nb, hkv, per)
        st["K"] = torch.empty((Nb * hkv * per, PAGE, d), dtype=torch.bfloat16, device=DEV)
        st["V"] = torch.empty_like(st["K"])
        st["K"][order] = K.reshape(-1, PAGE, d)
        st["V"][order] = V.reshape(-1, PAGE, d)
    elif case["kind"] == "prompt":
        st["K"], st["V"] = torch.zeros_like(K), torch.zeros_like(V)
    else:
        st["K"], st["V"] = K, V
    return st


# ---- one pass ------------------------------------------------------------------------------------------------------

def _turn(x, positions, freq, axis, pairs, adjacent, inverse):
    # (angles in 64 bits: a far position times a frequency has no bits left for the turn in 32)
    angle = positions[axis.long()].permute(1, 2, 0).double() * freq.double()
    cos, sin = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if inverse:
        sin = -sin
    y = x.float()
    if adjacent:
        a, b = y[..., 0:2 * pairs:2], y[..., 1:2 * pairs:2]
    else:
        a, b = y[..., :pairs], y[..., pairs:2 * pairs]
    a, b = a * cos - b * sin, b * cos + a * sin
    both = torch.stack((a, b), dim=-1).flatten(-2) if adjacent else torch.cat((a, b), dim=-1)
    return torch.cat((both, y[..., 2 * pairs:]), dim=-1).to(torch.bfloat16)


def _attention(st, K, V, received):
    """K, V [B][hkv][capacity][d], the chunk's rows behind the cached ones."""
    case, q = st["case"], st["q"]
    Nb, T, hq, d = q.shape
    hkv = K.shape[1]
    G = hq // hkv
    rows = case["cached"] + case["tokens"]
    K, V = K[:, :, :rows].float(), V[:, :, :rows].float()
    slot = torch.arange(rows, device=q.device)
    token = torch.arange(T, device=q.device)
    total = st["n_old"] + st["n_new"]
    in_use = slot < total[:, None]                                                 # [B][rows]
    valid = token < st["n_new"][:, None]                                           # [B][T]
    x = torch.matmul(q.float().reshape(Nb, T, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(Nb * hkv, G * T, d),
                     K.reshape(Nb * hkv, rows, d).transpose(1, 2)) * (1.0 / math.sqrt(d))
    x = x.reshape(Nb, hkv, G, T, rows)
    if case["kind"] == "shaped":
        own_pos, pos = st["own_pos"][:, None, :, None], st["pos"][:, :, None, :]   # [B][.][T][.], [B][hkv][.][rows]
        lowest = own_pos - case["window"] + 1 if case["window"] else torch.full_like(own_pos, NEVER)
        if st["first"] is not None:
            lowest = torch.maximum(lowest, st["first"][:, None, :, None])
        highest = own_pos if st["last"] is None else st["last"][:, None, :, None]
        seen = (pos >= lowest) & (pos <= highest) & in_use[:, None, None]
        if case["cap"]:
            x = case["cap"] * torch.tanh(x / case["cap"])
        if st["slope"] is not None:
            x = x - st["slope"].reshape(1, hkv, G, 1, 1) * (own_pos - pos).abs().float()[:, :, None]
        x = x.masked_fill(~seen[:, :, None], -math.inf)
    else:
        seen = slot <= st["n_old"][:, None, None] + token[:, None]                 # [B][T][rows]
        x = x.masked_fill(~(seen & in_use[:, None])[:, None, None], -math.inf)
    top = x.max(dim=-1, keepdim=True).values
    p = torch.exp(x - top)
    l = p.sum(dim=-1, keepdim=True)
    p = p / l
    o = torch.matmul(p.reshape(Nb * hkv, G * T, rows), V.reshape(Nb * hkv, rows, d)).reshape(Nb, hkv, G, T, d)
    out = torch.where(valid[:, :, None, None], o.permute(0, 3, 1, 2, 4).reshape(Nb, T, hq, d), 0.0).to(torch.bfloat16)
    lse = torch.where(valid[:, :, None], (top + torch.log(l))[..., 0].permute(0, 3, 1, 2).reshape(Nb, T, hq), 0.0)
    if not received:
        return dict(out=out, lse=lse)
    got = torch.where(valid[:, None, None, :, None], p, 0.0).sum(dim=(2, 3)) * in_use[:, None]
    full = torch.zeros((Nb, hkv, st["capacity"]), dtype=torch.float32, device=q.device)
    full[:, :, :rows] = got
    return dict(out=out, lse=lse, received=full)


def run(st):
    case = st["case"]
    if case["kind"] == "rotate":
        if own:
            from paper_2601_18383_amd import binding as B
            B.dynts_rotate(st["rotary"], st["q"], st["k"], st["positions"], st["q_out"], st["k_out"], inverse=case["inverse"])
            return dict(q=st["q_out"], k=st["k_out"])
        how = (st["positions"], st["freq"], st["axis"], case["pairs"], case["adjacent"], case["inverse"])
        return dict(q=_turn(st["q"], *how), k=_turn(st["k"], *how))
    if own:
        from paper_2601_18383_amd import binding as B
        c = st["cache"]
        if case["kind"] == "prompt":
            # a new request takes the place of the last one
            c.seq_len.zero_()
            c.next_pos.zero_()
            B.dynts_chunk_step(c.ctx, 0, st["q"], st["k_new"], st["v_new"], st["out"], st["scratch"], lse=st["lse"],
                               n_new=st["n_new"], question=True)
            return dict(out=st["out"], lse=st["lse"], K=c.K[0], V=c.V[0], length=c.seq_len)
        shaping = st.get("shaping")
        B.dynts_chunk_attend(c.ctx, 0, st["q"], st["out"], st["scratch"], lse=st["lse"], n_new=st["n_new"], shaping=shaping)
        if case["kind"] != "score":
            return dict(out=st["out"], lse=st["lse"])
        B.dynts_chunk_scores(c.ctx, 0, st["q"], st["lse"], dst=st["received"], accumulate=False, n_new=st["n_new"])
        return dict(out=st["out"], lse=st["lse"], received=st["received"])
    if case["kind"] == "prompt":
        T = case["tokens"]
        new = (torch.arange(T, device=DEV) < st["n_new"][:, None])[:, None, :, None]
        st["K"][:, :, :T] = torch.where(new, st["k_new"].transpose(1, 2), st["K"][:, :, :T])
        st["V"][:, :, :T] = torch.where(new, st["v_new"].transpose(1, 2), st["V"][:, :, :T])
        got = _attention(st, st["K"], st["V"], False)
        return dict(got, K=st["K"], V=st["V"], length=st["n_new"].reshape(1, -1).clone())
    K, V = st["K"], st["V"]
    if case["paged"]:
        K, V = K[st["table"]].flatten(2, 3), V[st["table"]].flatten(2, 3)
    return _attention(st, K, V, case["kind"] == "score")


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def _pairs(case):
    """Pairs of a query token and a key that it sees, over the batch (a mean where lengths differ)."""
    T, n, B = case["tokens"], case["cached"], case["batch"]
    if case["ragged"]:
        one = 1 if B == 1 else (1 + (B - 1) * (2 / 3)) / B
        n *= one
        T *= 1 if B == 1 else (1 + (B - 1) * 0.5) / B
    if case["documents"]:
        span = (n + T) / (case["documents"] + 1)
        return B * T * min(n + T / 2, span)
    if case["window"]:
        share = (n + T) / max(1.0, n + T + case["gaps"])
        return B * T * min(n + T / 2, case["window"] * share)
    both = case["prefix"] * case["prefix"] / 2 if case["prefix"] else 0
    return B * (T * n + T * (T + 1) / 2 + both)


def work(case):
    B, T, hq, hkv, d = case["batch"], case["tokens"], case["hq"], case["hkv"], case["d"]
    if case["kind"] == "rotate":
        heads = B * T * (hq + hkv)
        return {"bytes": 2 * heads * d * 2 + 4 * case["axes"] * B * T, "flops": 6 * heads * case["pairs"]}
    pairs = _pairs(case)
    n = case["cached"]
    new, old = (T * 0.5, n * 2 / 3) if case["ragged"] and B > 1 else (T, n)
    seen = old + new
    if case["window"]:
        seen = min(seen, (case["window"] + new) * (n + T) / (n + T + case["gaps"]))
    nbytes = B * (2 * new * hq * d * 2 + 4 * new * hq + 2 * seen * hkv * d * 2)
    flops = 4 * d * hq * pairs
    if case["kind"] == "prompt":
        nbytes += B * 2 * new * hkv * d * 2
    if case["kind"] == "score":
        nbytes += B * 4 * hkv * seen
        flops += 2 * hq * pairs
    if case["kind"] == "shaped":
        nbytes += B * 4 * hkv * seen
    return {"bytes": int(nbytes), "flops": int(flops)}


# ---- the definition, in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "rotate":
        x = _rotate_inputs(case, seed)
        P = case["pairs"]
        got = {}
        for name in ("q", "k"):
            y = x[name].double()
            for p in range(P):
                i, j = (2 * p, 2 * p + 1) if case["adjacent"] else (p, P + p)
                theta = x["positions"][int(x["axis"][p])].double() * float(x["freq"][p])
                z = torch.polar(torch.ones_like(theta), -theta if case["inverse"] else theta)[..., None]
                turned = torch.complex(y[..., i], y[..., j]) * z
                y[..., i], y[..., j] = turned.real, turned.imag
            got[name] = y
        return got
    x = _chunk_inputs(case, seed)
    Nb, hq, hkv, d, T = case["batch"], case["hq"], case["hkv"], case["d"], case["tokens"]
    capacity = (case["cached"] + T + PAGE - 1) // PAGE * PAGE
    out = torch.zeros((Nb, T, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((Nb, T, hq), dtype=torch.float64, device=DEV)
    received = torch.zeros((Nb, hkv, capacity), dtype=torch.float64, device=DEV)
    n_old, n_new = x["n_old"].tolist(), x["n_new"].tolist()
    for b in range(Nb):
        m, end = n_new[b], n_old[b] + n_new[b]
        if m == 0:
            continue
        at = torch.arange(n_old[b], end, device=DEV)
        for h in range(hq):
            g = h // (hq // hkv)
            s = x["q"][b, :m, h].double() @ x["k"][b, :end, g].double().t() / math.sqrt(d)
            hidden = torch.arange(end, device=DEV)[None] > at[:, None]
            if case["kind"] == "shaped":
                keys = x["pos"][b, g, :end].long()
                mine = x["own_pos"][b, :m].long()
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if x["slope"] is not None:
                    s = s - float(x["slope"][h]) * (mine[:, None] - keys).abs().double()
                high = mine if x["last"] is None else x["last"][b, :m].long()
                hidden = keys > high[:, None]
                if x["first"] is not None:
                    hidden |= keys < x["first"][b, :m].long()[:, None]
                if case["window"]:
                    hidden |= keys <= (mine - case["window"])[:, None]
            s[hidden] = -math.inf
            lse[b, :m, h] = torch.logsumexp(s, dim=-1)
            w = torch.exp(s - lse[b, :m, h][:, None])
            out[b, :m, h] = w @ x["v"][b, :end, g].double()
            if case["kind"] == "score":
                received[b, g, :end] += w.sum(dim=0)
    if case["kind"] == "score":
        return dict(out=out, lse=lse, received=received)
    if case["kind"] != "prompt":
        return dict(out=out, lse=lse)
    # (rows of the cache and lengths are copies, not computed numbers)
    return dict(out=out, lse=lse, K=None, V=None, length=None)
