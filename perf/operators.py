"""Performance cases of an uncompressed attention layer's operators.

STAR-KV leaves some layers uncompressed.  Such a layer rotates queries and keys, keeps keys and
values at 8 bits with a scale for each block of tokens and KV head, attends over them, and
shortens its cache by the attention weight that its blocks have gathered.  A case is one pass
through one of these operators:

  rope    rotary positions of query and key heads that lie in fused projection rows
  append  new keys and values into the 8-bit cache, and the rows that they touch read back
  attend  attention of one or more query tokens per sequence over the cache
  evict   choice of the blocks that stay, written to a new block table

``run`` computes them in plain torch (``own`` false) or through the library (``own`` true);
``exact`` is the same result in float64.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
TOP = {"int8": 127.0, "e4m3": 448.0}


def _rope(name, batch, n, heads, d, rotary, layout, scaling, dtype, far, theta=5e5, factor=8.0,
          inverse=False):
    """far: positions are below it; heads: query and key heads rotated together."""
    return {"name": name, "kind": "rope", "batch": batch, "n": n, "heads": heads, "d": d,
            "rotary": rotary, "layout": layout, "scaling": scaling, "dtype": dtype, "far": far,
            "theta": theta, "factor": factor, "inverse": inverse}


def _append(name, batch, n, n_kv, d, code, T, dtype, lo, hi, ragged=False):
    """lo..hi: tokens that the cache holds before; ragged: fewer than n new ones in some rows."""
    return {"name": name, "kind": "append", "batch": batch, "n": n, "n_kv": n_kv, "d": d,
            "code": code, "T": T, "dtype": dtype, "lo": lo, "hi": hi, "ragged": ragged}


def _attend(name, batch, n, n_q, n_kv, d, code, T, dtype, lo, hi, weights=False, ragged=False):
    """lo..hi: tokens in the cache, the n query tokens among them; weights: gathered per block;
    ragged: fewer than n query tokens in some sequences (a padded batch)."""
    return {"name": name, "kind": "attend", "batch": batch, "n": n, "n_q": n_q, "n_kv": n_kv,
            "d": d, "code": code, "T": T, "dtype": dtype, "lo": lo, "hi": hi, "weights": weights,
            "ragged": ragged}


def _evict(name, batch, n_kv, T, lo, hi, keep, sink, recent):
    """lo..hi: tokens in the cache; keep, sink, recent: blocks."""
    return {"name": name, "kind": "evict", "batch": batch, "n_kv": n_kv, "T": T, "lo": lo,
            "hi": hi, "keep": keep, "sink": sink, "recent": recent}


def listed():
    return [
        # a decode step of eight conversations: 32 query and 8 key heads of each new token
        _rope("rope_step_8x1_bf16", 8, 1, 40, 128, 128, "half", "plain", "bf16", 131072),
        # prompts of an 8B layer whose context was extended by bands of wavelengths
        _rope("rope_prompt_4x4096_bands_bf16", 4, 4096, 40, 128, 128, "half", "bands", "bf16",
              131072),
        # the gradient of a rotation of neighbouring pairs in three quarters of the head, odd sizes
        _rope("rope_back_3x1501_part_yarn_f16", 3, 1501, 7, 128, 96, "interleaved", "yarn", "f16",
              40000, theta=1e4, factor=16.0, inverse=True),
        # continuous batching: one token appended to each of 32 ragged sequences
        _append("append_step_32x1_int8", 32, 1, 8, 128, "int8", 64, "bf16", 2047, 16383),
        # two prompts of odd length after a cached prefix, 8-bit floating point
        _append("append_prompt_2x4099_e4m3", 2, 4099, 8, 128, "e4m3", 32, "bf16", 0, 40),
        # smallest call: one short sequence, no shared heads; launch latency counts
        _attend("attend_1x1000_d64_int8", 1, 1, 4, 1, 64, "int8", 64, "f16", 1000, 1000),
        # the long-context decode step: 4 x 128K
        _attend("attend_4x128k_int8", 4, 1, 32, 8, 128, "int8", 64, "bf16", 131072, 131072),
        # continuous batching with weights gathered for eviction
        _attend("attend_32x_ragged_e4m3_weights", 32, 1, 32, 8, 128, "e4m3", 32, "bf16", 2048,
                16384, weights=True),
        # five drafted tokens verified at a time in a 70B layer
        _attend("attend_draft5_2x64k_int8", 2, 5, 64, 8, 128, "int8", 128, "bf16", 65533, 65536),
        # a chunk of a long prompt against what is cached
        _attend("attend_chunk512_1x32k_int8", 1, 512, 32, 8, 128, "int8", 64, "bf16", 32768, 32768),
        # a prompt's cache shortened to a quarter after it was read
        _evict("evict_4x128k_t64", 4, 8, 64, 131072, 131072, 512, 1, 8),
        # ragged sequences in small blocks
        _evict("evict_32x_ragged_t16", 32, 8, 16, 2048, 16384, 200, 4, 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["rope", "append", "attend", "attend", "evict"])
    batch = _log_int(rng, 1, 40)
    d = rng.choice([64, 128, 128])
    n_kv = rng.choice([1, 2, 4, 8, 8])
    T = rng.choice([16, 32, 64, 128])
    code = rng.choice(["int8", "e4m3"])
    dtype = rng.choice(["f16", "bf16", "bf16"])
    if kind == "rope":
        heads = rng.randint(1, 72)
        n = _log_int(rng, 1, max(1, 600000 // (batch * heads)))
        c = _rope("", batch, n, heads, d, rng.choice([d, d, d // 2, 2 * rng.randint(2, d // 2)]),
                  rng.choice(["half", "interleaved"]),
                  rng.choice(["plain", "linear", "ntk", "bands", "yarn"]),
                  rng.choice(["f16", "bf16", "f32"]), _log_int(rng, 64, 1000000),
                  theta=rng.choice([1e4, 5e5]), factor=rng.choice([2.0, 8.0, 32.0]),
                  inverse=rng.random() < 0.3)
    elif kind == "append":
        n = _log_int(rng, 1, max(1, 60000 // (batch * n_kv)))
        lo = rng.randint(0, 300)
        c = _append("", batch, n, n_kv, d, code, T, dtype, lo, lo + rng.randint(0, 500),
                    ragged=rng.random() < 0.5)
    elif kind == "attend":
        n_q = n_kv * rng.choice([1, 2, 3, 4, 8])
        n = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 400)])
        # at most a quarter of the largest listed case's cache, of the chunk's scores
        top = min(131072, (1 << 20) // (batch * n_kv), (1 << 25) // (batch * n * n_q))
        hi = _log_int(rng, n, max(n, top))
        lo = hi if rng.random() < 0.3 else rng.randint(0, hi)
        c = _attend("", batch, n, n_q, n_kv, d, code, T, dtype, lo, hi,
                    weights=n * (n_q // n_kv) <= 64 and rng.random() < 0.5,
                    ragged=n > 1 and rng.random() < 0.5)
    else:
        hi = _log_int(rng, 64, 131072)
        keep = _log_int(rng, 2, max(2, hi // T))
        sink = rng.randint(0, keep // 2)
        c = _evict("", batch, n_kv, T, rng.randint(hi // 8, hi), hi, keep, sink,
                   rng.randint(0, keep - sink))
    del c["name"]
    return c


# ------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * (seed % 4000037) + 29)
    return g


def _lengths(c, g, lo, hi):
    return torch.randint(lo, hi + 1, (c["batch"],), generator=g, device="cuda").to(torch.int32)


def _rows(c, g, n, first, count):
    """Heads first..first+count of fused projection rows [batch][n][..][d]: a strided view."""
    x = torch.randn((c["batch"], n, first + count + 3, c["d"]), generator=g, device="cuda",
                    dtype=TYPES[c["dtype"]])
    return x[:, :, first:first + count]


def _rope_inputs(c, g):
    x = _rows(c, g, c["n"], 0, c["heads"])
    pos = torch.randint(0, c["far"], (c["batch"], 1), generator=g, device="cuda")
    pos = pos + torch.arange(c["n"], device="cuda")
    return x, pos.to(torch.int32)


def _kv(c, g, n, first=0):
    """New keys and values: normal, with a few key channels eight times larger, as models have."""
    k, v = _rows(c, g, n, first, c["n_kv"]), _rows(c, g, n, first, c["n_kv"])
    loud = torch.randperm(c["d"], generator=g, device="cuda")[:c["d"] // 32]
    k[..., loud] *= 8.0
    return k, v


def _append_inputs(c, g):
    """(keys and values of the unfinished block's earlier tokens, new keys and values, tokens
    held before, new tokens per sequence)."""
    pos = _lengths(c, g, c["lo"], c["hi"])
    n_new = torch.full_like(pos, c["n"])
    if c["ragged"]:
        n_new = _lengths(c, g, 0, c["n"])
    return _kv(c, g, c["T"]), _kv(c, g, c["n"], 5), pos, n_new


def _attend_inputs(c, g):
    k, v = _kv(c, g, c["hi"])
    q = _rows(c, g, c["n"], 0, c["n_q"])
    ctx = _lengths(c, g, c["lo"], c["hi"])
    q_len = torch.full_like(ctx, c["n"])
    if c["ragged"]:
        q_len = _lengths(c, g, 0, c["n"])
    blocks = -(-c["hi"] // c["T"])
    w = torch.rand((c["batch"], c["n_kv"], blocks), generator=g, device="cuda")
    return k, v, q, ctx, q_len, w


def _evict_inputs(c, g):
    """Weights as attention leaves them (a few blocks hold most), some of them equal."""
    blocks = -(-c["hi"] // c["T"])
    shape = (c["batch"], c["n_kv"], blocks)
    w = torch.exp(2.0 * torch.randn(shape, generator=g, device="cuda"))
    w = torch.where(torch.rand(shape, generator=g, device="cuda") < 0.1, torch.round(w), w)
    n = c["batch"] * c["n_kv"] * blocks
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(shape)
    return w, table, _lengths(c, g, c["lo"], c["hi"])


def _own_layer(c, capacity, n_q, table=None):
    from paper_2606_08382_amd import starkv as S
    from paper_2606_08382_amd.device import DenseLayer
    return DenseLayer(c["batch"], n_q, c["n_kv"], c.get("d", 128), capacity,
                      code=S.CODE_E4M3 if c.get("code") == "e4m3" else S.CODE_INT8,
                      block_tokens=c["T"],
                      dtype=S.DT_BF16 if c.get("dtype", "bf16") == "bf16" else S.DT_F16,
                      block_table=table)


def _own_rope(c):
    from paper_2606_08382_amd import starkv as S
    from paper_2606_08382_amd.device import Rope
    dtype = {"f16": S.DT_F16, "bf16": S.DT_BF16, "f32": S.DT_F32}[c["dtype"]]
    layout = S.ROPE_HALF if c["layout"] == "half" else S.ROPE_INTERLEAVED
    scaling = {"plain": S.ROPE_PLAIN, "linear": S.ROPE_LINEAR, "ntk": S.ROPE_NTK,
               "bands": S.ROPE_BANDS, "yarn": S.ROPE_YARN}[c["scaling"]]
    return Rope(c["d"], c["theta"], rotary_dim=c["rotary"], layout=layout, scaling=scaling,
                factor=c["factor"], original_ctx=8192, dtype=dtype)


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = {"c": c}
    if c["kind"] == "rope":
        x, pos = _rope_inputs(c, g)
        st.update(x=x, pos=pos, out=torch.empty(x.shape, dtype=x.dtype, device="cuda"))
        if own:
            st["rope"] = _own_rope(c)
    elif c["kind"] == "append":
        (k0, v0), (k, v), pos, n_new = _append_inputs(c, g)
        T, n = c["T"], c["n"]
        rows = (c["batch"], n + T - 1, c["n_kv"], c["d"])
        st.update(k=k, v=v, pos=pos, n_new=n_new, k0=k0, v0=v0, start=pos // T * T, end=pos + n_new,
                  k_out=torch.empty(rows, device="cuda"), v_out=torch.empty(rows, device="cuda"))
        if own:
            st["layer"] = _own_layer(c, c["hi"] + n, c["n_kv"])
            # what the cache holds of the block that the first new token falls in
            st["layer"].append(k0, v0, st["start"], n_new=pos % T)
    elif c["kind"] == "attend":
        k, v, q, ctx, q_len, w = _attend_inputs(c, g)
        st.update(q=q, ctx=ctx, q_len=q_len, w=w if c["weights"] else None,
                  out=torch.zeros((c["batch"], c["n"], c["n_q"], c["d"]), dtype=q.dtype,
                                  device="cuda"))
        if own:
            st["layer"] = _own_layer(c, c["hi"], c["n_q"])
            st["layer"].append(k, v, torch.zeros_like(ctx), n_new=ctx)
        else:
            st["kc"], st["ks"], st["kt"] = _plain_cache(c, k, ctx)
            st["vc"], st["vs"], st["vt"] = _plain_cache(c, v, ctx)
    else:
        w, table, ctx = _evict_inputs(c, g)
        st.update(w=w, table=table, ctx=ctx, table_out=torch.empty_like(table),
                  w_out=torch.empty_like(w), ctx_out=torch.empty_like(ctx))
        if own:
            st["layer"] = _own_layer({**c, "d": 64}, c["hi"], c["n_kv"], table=table)
    return st


# ------------------------------------------------------------------------------- plain form

def _freq(c):
    """Rotary frequencies of the pairs and the factor on cos and sin."""
    R, s, L0 = c["rotary"], c["factor"], 8192.0
    j = torch.arange(R // 2, device="cuda", dtype=torch.float64)
    f = c["theta"] ** (-2.0 * j / R)
    if c["scaling"] == "linear":
        return f / s, 1.0
    if c["scaling"] == "ntk":
        return (c["theta"] * s ** (R / (R - 2.0))) ** (-2.0 * j / R), 1.0
    if c["scaling"] == "bands":
        w = ((L0 * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return f * (w + (1.0 - w) / s), 1.0
    if c["scaling"] == "yarn":
        at = [R * math.log(L0 / (2 * math.pi * turns)) / (2 * math.log(c["theta"]))
              for turns in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), R - 1)
        ramp = ((j - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        return f * (1.0 - ramp) + f / s * ramp, 0.1 * math.log(s) + 1.0
    return f, 1.0


def _plain_rope(c, x, pos, out):
    f, m = _freq(c)
    R = c["rotary"]
    ang = torch.remainder(pos.double()[..., None] * f, 2 * math.pi).float()[:, :, None]
    cs, sn = torch.cos(ang) * m, torch.sin(ang) * m
    if c["inverse"]:
        sn = -sn
    y = x.float()
    if c["layout"] == "half":
        a, b = y[..., :R // 2], y[..., R // 2:R]
        z = torch.cat([a * cs - b * sn, b * cs + a * sn], dim=-1)
    else:
        a, b = y[..., 0:R:2], y[..., 1:R:2]
        z = torch.stack([a * cs - b * sn, b * cs + a * sn], dim=-1).flatten(-2)
    out.copy_(torch.cat([z, y[..., R:]], dim=-1))
    return out


def _plain_quantize(c, x):
    """Codes (as numbers, in float32) and scales of blocks [..., T, d]; the quotient in 64 bits,
    where a value next to a border between two codes is decided."""
    top = torch.full((1, 1), TOP[c["code"]], dtype=torch.float64, device="cuda")
    s = (x.abs().amax((-2, -1), keepdim=True).double() / top).float()
    r = x.double() / torch.where(s > 0, s, 1.0).double()
    if c["code"] == "int8":
        r = torch.round(r)
    else:
        step = torch.exp2(torch.clamp(torch.frexp(r)[1] - 1, min=-6).double() - 3)
        r = torch.round(r / step) * step
    r = torch.clamp(r, -TOP[c["code"]], TOP[c["code"]])
    return torch.where(s > 0, r.float(), 0.0), s


def _plain_cache(c, x, ctx):
    """Codes [B][H][blocks][T][d] and scales [B][H][blocks] of a sequence's tokens, and the 16-bit
    rows of its unfinished block."""
    T = c["T"]
    blocks = x.shape[1] // T + 1
    x = x.permute(0, 2, 1, 3)
    x = torch.nn.functional.pad(x, (0, 0, 0, blocks * T - x.shape[2]))
    x = x.reshape(x.shape[0], x.shape[1], blocks, T, c["d"])
    parts = [_plain_quantize(c, x[:, h:h + 1]) for h in range(c["n_kv"])]
    dt = torch.int8 if c["code"] == "int8" else torch.float8_e4m3fn
    codes = torch.cat([p[0].to(dt) for p in parts], dim=1)
    scales = torch.cat([p[1] for p in parts], dim=1)
    last = (ctx.long() // T)[:, None, None, None, None].expand(-1, c["n_kv"], 1, T, c["d"])
    return codes, scales[..., 0, 0], torch.gather(x, 2, last)[:, :, 0]


def _plain_append(c, st, x0, x, out):
    T, n, B = c["T"], c["n"], c["batch"]
    blocks = (n + 2 * T - 2) // T
    off = (st["pos"] - st["start"]).long()
    r = torch.arange(blocks * T, device="cuda")
    # row r of the touched blocks: an earlier token, a new one, or none yet
    old = r < off[:, None]
    new = ~old & (r < (off + st["n_new"])[:, None])
    idx = torch.where(old, r.expand(B, -1), r - off[:, None] + T)
    idx = torch.where(old | new, idx, 0)[:, :, None, None].expand(-1, -1, c["n_kv"], c["d"])
    y = torch.gather(torch.cat([x0, x], dim=1), 1, idx)
    y = torch.where((old | new)[:, :, None, None], y, 0.0).float()
    y = y.view(B, blocks, T, c["n_kv"], c["d"]).transpose(2, 3)
    codes, s = _plain_quantize(c, y)
    full = (torch.arange(1, blocks + 1, device="cuda") * T <= (off + st["n_new"])[:, None])
    y = torch.where(full[:, :, None, None, None], codes * s, y)
    out.copy_(y.transpose(2, 3).reshape(B, blocks * T, c["n_kv"], c["d"])[:, :n + T - 1])
    return out


def _plain_attend(c, st):
    B, H, T, d, n = c["batch"], c["n_kv"], c["T"], c["d"], c["n"]
    G = c["n_q"] // H
    ctx, q_len = st["ctx"].long(), st["q_len"].long()
    blocks = st["kc"].shape[2]
    is_last = (torch.arange(blocks, device="cuda") == (ctx // T)[:, None])[:, None, :, None, None]

    def values(codes, scales, tail):
        x = codes.float() * scales[..., None, None]
        return torch.where(is_last, tail[:, :, None].float(), x).view(B, H, blocks * T, d)

    K, V = values(st["kc"], st["ks"], st["kt"]), values(st["vc"], st["vs"], st["vt"])
    q = st["q"].float().view(B, n, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, d)
    s = torch.matmul(q, K.transpose(2, 3).contiguous()) / math.sqrt(d)
    j = torch.arange(n, device="cuda")
    seen = (ctx - q_len)[:, None] + j + 1                    # tokens that query token j sees
    live = j < q_len[:, None]
    seen = torch.where(live, seen, 0)
    mask = torch.arange(blocks * T, device="cuda") < seen[..., None]
    mask = mask[:, None, :, None].expand(B, 1, n, G, blocks * T).reshape(B, 1, n * G, blocks * T)
    s = torch.where(mask, s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    p = p / torch.clamp(p.sum(-1, keepdim=True), min=1e-30)
    o = torch.matmul(p, V).view(B, H, n, G, d).permute(0, 2, 1, 3, 4).reshape(B, n, H * G, d)
    st["out"].copy_(torch.where(live[..., None, None], o, st["out"].float()))
    if st["w"] is None:
        return st["out"]
    st["w"] += p.sum(2).view(B, H, blocks, T).sum(-1)[..., :st["w"].shape[2]]
    return st["out"], st["w"]


def _plain_evict(c, st):
    T, w, table = c["T"], st["w"], st["table"]
    blocks = w.shape[2]
    n = (st["ctx"].long() // T)[:, None, None]
    left = n - torch.clamp(n - c["keep"], min=0) // 2 * 2    # whole blocks that stay
    i = torch.arange(blocks, device="cuda").expand_as(w)
    must = (i < c["sink"]) | ((i >= n - c["recent"]) & (i < n))
    rank_key = torch.where(must, math.inf, torch.where(i < n, w, -math.inf))
    order = torch.argsort(rank_key, dim=-1, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(2, order, i)
    kept = (rank < left) & (i < n)
    # kept blocks in order, then those that leave, then the rest in place
    order = torch.argsort(torch.where(kept, 0, torch.where(i < n, 1, 2)), dim=-1, stable=True)
    st["table_out"].copy_(torch.gather(table, 2, order))
    moved = torch.gather(w, 2, torch.where(i == left, torch.clamp(n, max=blocks - 1), order))
    here = (i < left) | ((i == left) & (n < blocks))
    st["w_out"].copy_(torch.where(here, moved, 0.0))
    st["ctx_out"].copy_(st["ctx"] - ((n - left) * T)[:, 0, 0])
    return st["table_out"], st["w_out"], st["ctx_out"]


def run(state):
    st, c = state, state["c"]
    if c["kind"] == "rope":
        if own:
            return st["rope"](st["x"], st["pos"], out=st["out"], inverse=c["inverse"])
        return _plain_rope(c, st["x"], st["pos"], st["out"])
    if c["kind"] == "append":
        if own:
            if c["n"] > c["T"]:
                # an earlier pass took the unfinished block's 16-bit rows further: given again
                st["layer"].append(st["k0"], st["v0"], st["start"], n_new=st["pos"] - st["start"])
            st["layer"].append(st["k"], st["v"], st["pos"], n_new=st["n_new"])
            st["layer"].read(st["end"], st["start"], st["k_out"], st["v_out"])
            return st["k_out"], st["v_out"]
        return (_plain_append(c, st, st["k0"], st["k"], st["k_out"]),
                _plain_append(c, st, st["v0"], st["v"], st["v_out"]))
    if c["kind"] == "attend":
        if not own:
            return _plain_attend(c, st)
        o = st["layer"].attend(st["q"], st["ctx"], q_len=st["q_len"], weights=st["w"],
                               out=st["out"])
        return o if st["w"] is None else (o, st["w"])
    if own:
        return st["layer"].evict(st["w"], st["ctx"], c["keep"], sink=c["sink"],
                                 recent=c["recent"], table_out=st["table_out"],
                                 weights_out=st["w_out"], ctx_out=st["ctx_out"])
    return _plain_evict(c, st)


# ------------------------------------------------------------------------------- work

def work(case):
    c = case
    es = 4 if c.get("dtype") == "f32" else 2
    B = c["batch"]
    if c["kind"] == "rope":
        m = B * c["n"]
        return {"bytes": 2.0 * es * m * c["heads"] * c["d"] + 4 * m,
                "flops": 3.0 * m * c["heads"] * c["rotary"]}
    if c["kind"] == "append":
        rows = B * c["n"] * (0.5 if c["ragged"] else 1.0) * c["n_kv"] * c["d"] * 2
        back = B * (c["n"] + c["T"] - 1) * c["n_kv"] * c["d"] * 2
        # read at 16 bits, written at 8, read back and written at 32
        return {"bytes": rows * (es + 1) + back * (1.0 + 4.0), "flops": 4.0 * rows}
    if c["kind"] == "attend":
        tokens = B * (c["lo"] + c["hi"]) / 2
        share = 0.5 if c["ragged"] else 1.0
        nbytes = tokens * c["n_kv"] * 2 * (c["d"] + 4.0 / c["T"])
        nbytes += share * 2 * es * B * c["n"] * c["n_q"] * c["d"]
        if c["weights"]:
            nbytes += 8.0 * tokens / c["T"] * c["n_kv"]
        seen = max(tokens - B * (c["n"] - 1) / 2, B)
        return {"bytes": nbytes, "flops": share * 4.0 * seen * c["n"] * c["n_q"] * c["d"]}
    entries = B * c["n_kv"] * -(-c["hi"] // c["T"])
    return {"bytes": 16.0 * entries + 8 * B, "flops": 8.0 * entries}


# ------------------------------------------------------------------------------- exact

def _exact_rope(c, x, pos):
    R, s = c["rotary"], c["factor"]
    half = R // 2
    y = x.double().clone()
    gain = 0.1 * math.log(s) + 1.0 if c["scaling"] == "yarn" else 1.0
    theta = c["theta"]
    if c["scaling"] == "ntk":
        theta *= math.exp(math.log(s) * R / (R - 2))
    if c["scaling"] == "yarn":
        def where(turns):
            return math.log(8192.0 / (turns * 2 * math.pi)) / math.log(theta) * R / 2
        first, last = max(int(math.floor(where(32.0))), 0), min(int(math.ceil(where(1.0))), R - 1)
    for j in range(half):
        f = math.exp(-math.log(theta) * 2 * j / R)
        if c["scaling"] == "linear":
            f /= s
        elif c["scaling"] == "bands":
            turns = 8192.0 * f / (2 * math.pi)
            if turns <= 1.0:
                f /= s
            elif turns < 4.0:
                t = (turns - 1.0) / 3.0
                f = (1 - t) * f / s + t * f
        elif c["scaling"] == "yarn":
            t = min(max((j - first) / (last - first if last > first else 1e-3), 0.0), 1.0)
            f = t * f / s + (1 - t) * f
        a = (-1.0 if c["inverse"] else 1.0) * f * pos.double()[..., None]
        p, q = (j, j + half) if c["layout"] == "half" else (2 * j, 2 * j + 1)
        u, v = x[..., p].double(), x[..., q].double()
        y[..., p] = gain * (u * torch.cos(a) - v * torch.sin(a))
        y[..., q] = gain * (v * torch.cos(a) + u * torch.sin(a))
    return y


def _exact_block(c, x):
    """A block [..., T, d] after its round trip through 8 bits, float64."""
    x = x.double()
    top = TOP[c["code"]]
    s = (x.abs().flatten(-2).max(-1).values / torch.tensor(top, dtype=torch.float64,
                                                          device="cuda")).float().double()
    s = s[..., None, None]
    a = torch.where(s > 0, x.abs() / s, 0.0)
    if c["code"] == "int8":
        grid = torch.arange(128, device="cuda", dtype=torch.float64)
    else:
        e, m = torch.meshgrid(torch.arange(16), torch.arange(8), indexing="ij")
        grid = torch.where(e > 0, (8 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9.0).flatten()[:127]
        grid = grid.double().cuda()
    mid = (grid[1:] + grid[:-1]) / 2
    lo = torch.bucketize(a, mid)                 # borders below a
    hi = torch.bucketize(a, mid, right=True)     # borders at or below a
    even = torch.where(lo % 2 == 0, lo, hi)      # on a border: the even code
    return torch.sign(x) * grid[even] * s


def _exact_cache(c, x, n):
    """Rows [n][d] of one head as the cache stands for them, float64."""
    T = c["T"]
    f = n // T * T
    y = x[:n].double()
    if f:
        y[:f] = _exact_block(c, x[:f].reshape(f // T, T, c["d"])).view(f, c["d"])
    return y


def exact(case, seed):
    c, g = case, _gen(seed)
    if c["kind"] == "rope":
        return _exact_rope(c, *_rope_inputs(c, g))
    if c["kind"] == "append":
        old, new, pos, n_new = _append_inputs(c, g)
        got = []
        for x0, x in zip(old, new):
            y = torch.zeros((c["batch"], c["n"] + c["T"] - 1, c["n_kv"], c["d"]), device="cuda",
                            dtype=torch.float64)
            for b, (p, m) in enumerate(zip(pos.tolist(), n_new.tolist())):
                for h in range(c["n_kv"]):
                    rows = torch.cat([x0[b, :p % c["T"], h], x[b, :m, h]])
                    y[b, :len(rows), h] = _exact_cache(c, rows, len(rows))
            got.append(y)
        return tuple(got)
    if c["kind"] == "attend":
        k, v, q, ctx, q_len, w = _attend_inputs(c, g)
        o = torch.zeros(q.shape, device="cuda", dtype=torch.float64)
        w = w.double()
        G, T = c["n_q"] // c["n_kv"], c["T"]
        for b, (L, m) in enumerate(zip(ctx.tolist(), q_len.tolist())):
            if L == 0 or m == 0:
                continue
            seen = torch.arange(L - m + 1, L + 1, device="cuda").clamp(min=0)[:, None]
            mask = torch.arange(L, device="cuda") < seen
            for h in range(c["n_kv"]):
                K, V = _exact_cache(c, k[b, :, h], L), _exact_cache(c, v[b, :, h], L)
                for i in range(h * G, h * G + G):
                    s = (q[b, :m, i].double() @ K.T.contiguous()) / math.sqrt(c["d"])
                    p = torch.softmax(torch.where(mask, s, -math.inf), dim=-1)
                    p = torch.where(mask, p, 0.0)
                    o[b, :m, i] = p @ V
                    per = torch.zeros(w.shape[2] * T, device="cuda", dtype=torch.float64)
                    per[:L] = p.sum(0)
                    w[b, h] += per.view(-1, T).sum(-1)
        return (o, w) if c["weights"] else o
    w, table, ctx = (x.cpu() for x in _evict_inputs(c, g))
    t_out, w_out, c_out = table.clone(), torch.zeros_like(w), ctx.clone()
    for b, L in enumerate(ctx.tolist()):
        n = L // c["T"]
        gone = max(n - c["keep"], 0) // 2 * 2
        c_out[b] = L - gone * c["T"]
        for h in range(c["n_kv"]):
            ws = w[b, h].tolist()
            last = max(n - c["recent"], 0)
            free = [i for i in range(n) if c["sink"] <= i < last]
            free.sort(key=lambda i: (ws[i], -i))     # the lightest first, of equals the last
            out = set(free[:gone])
            order = [i for i in range(n) if i not in out] + sorted(out)
            t_out[b, h, :n] = table[b, h, order]
            w_out[b, h, :n - gone] = w[b, h, order[:n - gone]]
            if n < len(ws):
                w_out[b, h, n - gone] = w[b, h, n]
    return t_out.cuda(), w_out.double().cuda(), c_out.cuda()
