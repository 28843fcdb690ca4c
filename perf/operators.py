"""The K/V cache operators: appending with the rotation, the 8-bit cache, and the attention over it.

Three operators, each called through the public binding (``paper_2609_09338_gb300.binding``):

* ``osprey_kv_append_rope``: K/V rows into the bf16 paged cache, keys rotated on the way;
* ``osprey_kv8_append``: the same into the 8-bit cache, whose finished pages hold e4m3 codes with one scale for each
  page and head and whose unfinished page stays in a bf16 ring (the tail);
* ``osprey_kv8_attend``: causal attention of each sequence's newest rows over that cache.

``run`` computes them in elementary torch operations where ``own`` is false, and calls the binding where it is true.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BF, F32, F64, FP8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
PAGE = 16
THETA = 1e6
TYPES = {"bf16": BF, "f32": F32}


# ---------------------------------------------------------------- cases
def _append(name, kind, B, rows_lo, rows_hi, ctx_hi, L, Hq, Hkv, hd, dtype, advance, tail=2):
    """rows_lo..rows_hi new rows a sequence after 0..ctx_hi committed ones; L layers at once (advance) or one of them."""
    return {"name": name, "kind": kind, "B": B, "rows_lo": rows_lo, "rows_hi": rows_hi, "ctx_hi": ctx_hi, "L": L,
            "Hq": Hq, "Hkv": Hkv, "hd": hd, "dtype": dtype, "advance": advance, "tail": tail}


def _attend(name, B, rows_lo, rows_hi, ctx_lo, ctx_hi, Hq, Hkv, hd, dtype, rotate=False, advanced=True):
    """rows_lo..rows_hi query rows a sequence, the newest of ctx_lo..ctx_hi cached ones."""
    return {"name": name, "kind": "attend8", "B": B, "rows_lo": rows_lo, "rows_hi": rows_hi, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "Hq": Hq, "Hkv": Hkv, "hd": hd, "dtype": dtype, "rotate": rotate, "advanced": advanced}


def listed():
    return [
        # one decode step of a full server, one layer's rows taken out of the fused QKV projection: all latency
        _append("append-step-b64", "append", 64, 1, 1, 1000, 1, 16, 8, 128, "bf16", False),
        # prompts of a batch, every layer of a two-layer drafter at once
        _append("append-prompt-b16", "append", 16, 100, 4096, 0, 2, 16, 4, 128, "bf16", True),
        # float32 rows, small heads, odd counts, some sequences without a row
        _append("append-f32-b7", "append", 7, 0, 333, 77, 1, 4, 2, 64, "f32", False),
        # the decode step into the 8-bit cache: a page is finished every 16th time
        _append("append8-step-b64", "append8", 64, 1, 1, 1000, 1, 16, 8, 128, "bf16", False),
        # what a verification accepted: 1..8 rows of 96 sequences, float32
        _append("append8-accept-b96", "append8", 96, 1, 8, 500, 1, 16, 8, 128, "f32", False),
        # prompts into the 8-bit cache, both layers
        _append("append8-prompt-b16", "append8", 16, 100, 4096, 0, 2, 16, 4, 128, "bf16", True),
        # the smallest cache: three sequences of small heads that have just begun, nothing or one page in 8 bits
        _attend("attend8-begin-b3", 3, 1, 1, 1, 40, 4, 2, 64, "bf16"),
        # one stream, one token: the interactive step
        _attend("attend8-b1", 1, 1, 1, 2048, 2048, 16, 8, 128, "bf16", advanced=False),
        # a full server with long ragged contexts: bound by the cache's bytes
        _attend("attend8-b64-long", 64, 1, 1, 1024, 16384, 16, 8, 128, "bf16"),
        # float32 queries of groups of four, rotated on the way
        _attend("attend8-f32-b16", 16, 1, 1, 2048, 8192, 16, 4, 128, "f32", rotate=True),
        # ragged accepted rows of a batch share a sequence's keys
        _attend("attend8-rows8-b96", 96, 1, 8, 1024, 4096, 32, 8, 128, "bf16"),
        # blocks of 50..64 rows (block drafting, the nodes of a tree): compute begins to bind
        _attend("attend8-block64-b8", 8, 50, 64, 2000, 8192, 32, 8, 128, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append8", "attend8", "attend8"])
    hd, G = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8])
    Hkv = rng.choice([h for h in (1, 2, 4, 8) if h * G * hd % 256 == 0 and h * G <= 32])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "attend8":
        B = _log_int(rng, 1, 96)
        rows = rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 64)])
        # no more cached keys, and no more products, than the largest listed cases have
        most = min(16384, 64 * 8192 // B, 8 * 8192 * 64 // (B * rows))
        hi = _log_int(rng, 64, max(most, 65)) | rng.randint(0, 1)
        c = _attend("", B, rng.randint(0 if rows > 1 else 1, rows), rows, rng.randint(rows, max(rows, hi)), max(rows, hi), Hkv * G, Hkv,
                    hd, dtype, rng.random() < 0.5, rng.random() < 0.5)
    else:
        B = _log_int(rng, 1, 96)
        long = rng.random() < 0.4
        hi = _log_int(rng, 16, min(4096, 32768 // B)) if long else rng.randint(1, 17)
        c = _append("", kind, B, rng.randint(0, hi), hi, 0 if long else rng.randint(0, 900), rng.choice([1, 2]),
                    Hkv * G, Hkv, hd, dtype, long, rng.randint(2, 4))
    c.pop("name")
    return c


# ---------------------------------------------------------------- inputs
def _host_ints(case, seed):
    """Rows and committed lengths of every sequence (a program knows them when it plans the call): a case's own, in an
    order that goes by the seed."""
    names = ("B", "rows_lo", "rows_hi", "ctx_lo", "ctx_hi", "hd")
    g = torch.Generator().manual_seed(sum(31 ** i * case.get(k, 0) for i, k in enumerate(names)) % (1 << 40) + 13)
    B = case["B"]
    ints = lambda lo, hi: torch.randint(lo, hi + 1, (B,), generator=g).tolist()  # noqa: E731
    n, lens = ints(case["rows_lo"], case["rows_hi"]), ints(case.get("ctx_lo", 0), case["ctx_hi"])
    if case["kind"] == "attend8":
        lens = [max(t, r) for t, r in zip(lens, n)]
    elif not any(n):
        n[0] = 1
    order = torch.randperm(B, generator=torch.Generator().manual_seed(seed * 7919 + 13)).tolist()
    return [n[i] for i in order], [lens[i] for i in order]


def _keys(gen, shape):
    """Keys as a trained model has them: a few channels of each head are several times the others."""
    x = torch.randn(shape, generator=gen, device=DEV, dtype=BF)
    return x.mul_(torch.exp(0.5 * torch.randn(shape[-2:], generator=gen, device=DEV)).to(BF))


def _tables(lens, extra, gen):
    """Page tables of sequences that hold lens + extra rows, their pages in random order."""
    pages = [(n + e + PAGE - 1) // PAGE for n, e in zip(lens, extra)]
    total, most = max(1, sum(pages)), max(1, max(pages))
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros((len(lens), most), dtype=torch.int32, device=DEV)
    first = torch.cumsum(torch.tensor([0] + pages[:-1]), 0).to(DEV)
    slot = torch.arange(most, device=DEV)[None]
    have = slot < torch.tensor(pages, device=DEV)[:, None]
    table[have] = ids[(first[:, None] + slot)[have]]
    return table, total


def _context(case):
    """A drafter context of this case's heads (its projections are not part of these calls, so they are small)."""
    from paper_2609_09338_gb300 import binding as ob
    from paper_2609_09338_gb300.workloads import DrafterShape
    sh = DrafterShape(d_model=256, n_layers=case.get("L", 1), n_q_heads=case["Hq"], n_kv_heads=case["Hkv"],
                      head_dim=case["hd"], ffn_dim=256, vocab=256, feat_dim=256, rope_theta=THETA)
    z = lambda *s: torch.zeros(s, dtype=BF, device=DEV)  # noqa: E731
    d, a = sh.d_model, sh.n_q_heads * sh.head_dim
    w = {"W_c": z(d, sh.feat_dim), "embed": z(sh.vocab, d), "final_norm": z(d), "lm_head": z(sh.vocab, d)}
    for k, s in {"attn_norm": (d,), "W_qkv": (sh.qkv_rows, 2 * d), "W_o": (d, a), "ffn_norm": (d,),
                 "W_gate": (sh.ffn_dim, d), "W_up": (sh.ffn_dim, d), "W_down": (d, sh.ffn_dim)}.items():
        w[k] = [z(*s) for _ in range(sh.n_layers)]
    return ob.osprey_create(sh, w)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed * 1000003 + 17)
    B, Hq, Hkv, hd = case["B"], case["Hq"], case["Hkv"], case["hd"]
    dt = TYPES[case["dtype"]]
    n, lens = _host_ints(case, seed)
    s = {"case": case, "n_host": n, "lens_host": lens, "status": torch.zeros(1, dtype=torch.int32, device=DEV),
         "n_rows": torch.tensor(n, dtype=torch.int32, device=DEV)}
    if case["kind"] == "attend8":
        L = 1
        table, n_pages = _tables(lens, [0] * B, gen)
        s["max_rows"] = max(1, max(n))
        committed = lens if case["advanced"] else [t - r for t, r in zip(lens, n)]
        s["seq_len"] = torch.tensor(committed, dtype=torch.int32, device=DEV)
        tail = 2
        kv8 = {"k8": torch.empty((1, n_pages, Hkv, PAGE * hd), dtype=torch.uint8, device=DEV),
               "k_scale": torch.empty((1, n_pages, Hkv), dtype=F32, device=DEV)}
        kv8["v8"], kv8["v_scale"] = torch.empty_like(kv8["k8"]), torch.empty_like(kv8["k_scale"])
        chan = torch.exp(0.5 * torch.randn((Hkv, 1, hd), generator=gen, device=DEV)).to(BF)
        for p in range(0, n_pages, 4096):      # a part at a time: the values are several times their codes
            q = min(n_pages, p + 4096)
            x = torch.randn((1, q - p, Hkv, PAGE, hd), generator=gen, device=DEV, dtype=BF)
            kv8["k8"][:, p:q], kv8["k_scale"][:, p:q] = _encode(x * chan, False)
            x = torch.randn((1, q - p, Hkv, PAGE, hd), generator=gen, device=DEV, dtype=BF)
            kv8["v8"][:, p:q], kv8["v_scale"][:, p:q] = _encode(x, True)
        kv8["k_tail"] = torch.randn((1, B * tail, Hkv, PAGE, hd), generator=gen, device=DEV, dtype=BF) * chan
        kv8["v_tail"] = torch.randn((1, B * tail, Hkv, PAGE, hd), generator=gen, device=DEV, dtype=BF)
        # queries lie in rows of the fused QKV projection's output
        width = (Hq + 2 * Hkv) * hd
        s["qkv"] = torch.randn((B, s["max_rows"], width), generator=gen, device=DEV).to(dt)
        s["q"] = s["qkv"][..., :Hq * hd].unflatten(-1, (Hq, hd))
        s["out"] = torch.zeros((B, s["max_rows"], Hq, hd), dtype=dt, device=DEV)
    else:
        L = case["L"]
        table, n_pages = _tables(lens, n, gen)
        s["start"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["seq_len"] = s["start"].clone()
        tail = case["tail"]
        layers = L if case["advance"] else 1   # all layers of a prompt, or the one that the model is at
        total, width = sum(n), (Hq + 2 * Hkv) * hd
        s["total"] = total
        s["qkv"] = torch.randn((layers, total, width), generator=gen, device=DEV).to(dt)
        k = s["qkv"][..., Hq * hd:(Hq + Hkv) * hd].unflatten(-1, (Hkv, hd))
        k.mul_(torch.exp(0.5 * torch.randn((Hkv, hd), generator=gen, device=DEV)).to(dt))
        v = s["qkv"][..., (Hq + Hkv) * hd:].unflatten(-1, (Hkv, hd))
        s["k_rows"], s["v_rows"] = (k, v) if case["advance"] else (k[0], v[0])
        if case["kind"] == "append":
            s["k_pages"] = _keys(gen, (L, n_pages, Hkv, PAGE, hd)) if not case["advance"] else \
                torch.zeros((L, n_pages, Hkv, PAGE, hd), dtype=BF, device=DEV)
            s["v_pages"] = s["k_pages"].clone()
            kv8 = None
        else:
            kv8 = {"k8": torch.zeros((L, n_pages, Hkv, PAGE * hd), dtype=torch.uint8, device=DEV),
                   "v8": torch.zeros((L, n_pages, Hkv, PAGE * hd), dtype=torch.uint8, device=DEV),
                   "k_scale": torch.ones((L, n_pages, Hkv), dtype=F32, device=DEV),
                   "v_scale": torch.ones((L, n_pages, Hkv), dtype=F32, device=DEV),
                   "k_tail": _keys(gen, (L, B * tail, Hkv, PAGE, hd)),
                   "v_tail": _keys(gen, (L, B * tail, Hkv, PAGE, hd))}
    s["table"], s["tail"] = table, tail
    if kv8:
        s.update(kv8)
    if own:   # the handles that a program makes once: a context, and the cache's tensors together
        from paper_2609_09338_gb300 import binding as ob
        s["ctx"] = _context(case)
        s["kv"] = ob.Kv8Cache(**kv8, page_table=table, seq_len=s["seq_len"]) if kv8 else \
            ob.KvCache(s["k_pages"], s["v_pages"], table, s["seq_len"])
    return s


# ---------------------------------------------------------------- plain forms
def _rotate(x, pos):
    """Rotate-half at `pos` (one for each row) of x [..., rows, heads, hd], float32; angles in 64 bits."""
    h = x.shape[-1] // 2
    i = torch.arange(h, device=x.device, dtype=F64)
    a = pos.to(F64)[..., None] * torch.exp(i * (-2.0 * math.log(THETA) / x.shape[-1]))
    c, s = torch.cos(a).to(F32)[..., None, :], torch.sin(a).to(F32)[..., None, :]
    x1, x2 = x[..., :h], x[..., h:]
    return torch.cat([x1 * c - x2 * s, x2 * c + x1 * s], -1)


def _encode(x, values):
    """Blocks [..., 16, hd] of bf16 values as codes [..., 16 * hd] (uint8) and scales [...].

    The scale is the smallest power of two (2^-100 at least) that brings the block into e4m3's range.  Keys lie in
    groups of 8 slots, each of hd / 16 pieces of 8 slots x 16 dimensions; values have their 16 slots side by side."""
    hd = x.shape[-1]
    x = x.to(F32)
    m, e = torch.frexp(x.abs().amax((-2, -1)) / 448.0)
    e = torch.where(m > 0.5, e, e - 1).clamp_min(-100)
    e = torch.where(m > 0, e, torch.full_like(e, -100))
    scale = torch.ldexp(torch.ones_like(m), e)
    code = torch.ldexp(x, -e[..., None, None]).to(FP8).view(torch.uint8)
    if values:
        code = code.transpose(-1, -2)
    else:
        code = code.unflatten(-2, (2, 8)).unflatten(-1, (hd // 16, 16)).transpose(-3, -2)
    return code.reshape(*x.shape[:-2], PAGE * hd), scale


def _decode(code, scale, values):
    """The values [..., 16, hd] (float32) of codes and scales."""
    hd = code.shape[-1] // PAGE
    x = code.view(FP8).to(F32)
    if values:
        x = x.unflatten(-1, (hd, PAGE)).transpose(-1, -2)
    else:
        x = x.unflatten(-1, (2, hd // 16, 8, 16)).transpose(-3, -2).flatten(-4, -3).flatten(-2, -1)
    return x * scale[..., None, None]


def _rows_of(s):
    """Sequence and position of each new row."""
    n = s["n_rows"].to(torch.int64)
    seq = torch.repeat_interleave(torch.arange(len(s["n_host"]), device=DEV), n, output_size=s["total"])
    first = torch.cumsum(n, 0) - n
    return seq, s["seq_len"].to(torch.int64)[seq] + torch.arange(s["total"], device=DEV) - first[seq]


def _new_rows(s, pos):
    """The rows as they are cached: [layers, total, Hkv, hd] bf16."""
    k, v = s["k_rows"], s["v_rows"]
    if k.dim() == 3:
        k, v = k[None], v[None]
    return _rotate(k.to(F32), pos).to(BF), v.to(BF)


def _plain_append(s):
    seq, pos = _rows_of(s)
    k, v = _new_rows(s, pos)
    page = s["table"][seq, pos // PAGE].to(torch.int64)
    s["k_pages"][:k.shape[0], page, :, pos % PAGE] = k.transpose(0, 1)
    s["v_pages"][:v.shape[0], page, :, pos % PAGE] = v.transpose(0, 1)


def _plain_append8(s):
    T = s["tail"]
    start, n = s["seq_len"].to(torch.int64), s["n_rows"].to(torch.int64)
    seq, pos = _rows_of(s)
    k, v = _new_rows(s, pos)
    L = k.shape[0]
    # pages that these rows finish: their rows, older ones from the tail
    done = (start + n) // PAGE - start // PAGE
    total = sum((a + b) // PAGE - a // PAGE for a, b in zip(s["lens_host"], s["n_host"]))
    b = torch.repeat_interleave(torch.arange(len(s["n_host"]), device=DEV), done, output_size=total)
    p = start[b] // PAGE + torch.arange(total, device=DEV) - (torch.cumsum(done, 0) - done)[b]
    at = p[:, None] * PAGE + torch.arange(PAGE, device=DEV)
    old = at < start[b][:, None]
    row = ((torch.cumsum(n, 0) - n)[b][:, None] + at - start[b][:, None]).clamp_min(0)
    ids = s["table"][b, p].to(torch.int64)
    for new, name, values in ((k, "k", False), (v, "v", True)):
        before = s[name + "_tail"][:L, b * T + p % T]
        block = torch.where(old[None, :, None, :, None], before, new[:, row].transpose(2, 3))
        s[name + "8"][:L, ids], s[name + "_scale"][:L, ids] = _encode(block, values)
    # the tail keeps the rows of the last pages
    last = (start + n - 1) // PAGE
    keep = torch.where(pos // PAGE > last[seq] - T, seq * T + pos // PAGE % T, torch.full_like(pos, -1))
    for new, name in ((k, "k_tail"), (v, "v_tail")):
        buf, spare = s[name], torch.zeros_like(s[name][:, :1])
        both = torch.cat([buf, spare], 1)   # rows that are not kept go to a page of their own
        both[:L, torch.where(keep >= 0, keep, torch.full_like(keep, buf.shape[1])), :, pos % PAGE] = new.transpose(0, 1)
        buf.copy_(both[:, :-1])


def _plain_attend(s):
    c = s["case"]
    B, R, Hq, Hkv, hd = c["B"], s["max_rows"], c["Hq"], c["Hkv"], c["hd"]
    n = s["n_rows"].to(torch.int64)
    total = s["seq_len"].to(torch.int64) + (0 if c["advanced"] else n)
    c8 = total // PAGE
    P8 = max(t // PAGE for t in s["lens_host"])
    ids = s["table"][:, :P8].to(torch.int64)
    at = torch.arange(P8 * PAGE + PAGE, device=DEV)
    ring = torch.arange(B, device=DEV) * s["tail"] + c8 % s["tail"]
    at = torch.where(at < P8 * PAGE, at, at - P8 * PAGE + c8[:, None] * PAGE)
    held = torch.cat([at[:, :P8 * PAGE] < c8[:, None] * PAGE, at[:, P8 * PAGE:] < total[:, None]], 1)
    parts = []
    for name, values in (("k", False), ("v", True)):
        x = _decode(s[name + "8"][0, ids], s[name + "_scale"][0, ids], values)      # [B, P8, Hkv, 16, hd]
        x = x.transpose(1, 2).reshape(B, Hkv, P8 * PAGE, hd)
        x = torch.cat([x, s[name + "_tail"][0, ring].to(F32)], 2)
        parts.append(torch.where(held[:, None, :, None], x, torch.zeros_like(x)))
    j = torch.arange(R, device=DEV)
    qpos = (total - n)[:, None] + j
    q = s["q"].to(F32)
    if c["rotate"]:
        q = _rotate(q, qpos)
    q = q.reshape(B, R, Hkv, Hq // Hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, hd)
    score = torch.matmul(q, parts[0].transpose(-1, -2)) / math.sqrt(hd)
    see = held[:, None] & (at[:, None] <= qpos[:, :, None])                          # [B, R, keys]
    see = see.repeat_interleave(Hq // Hkv, 1)[:, None]
    score = torch.where(see, score, torch.full_like(score, -math.inf))
    live = (j[None] < n[:, None])
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    o = torch.matmul(w, parts[1]) / w.sum(-1, keepdim=True)
    o = o.reshape(B, Hkv, R, Hq // Hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, R, Hq, hd).to(s["out"].dtype)
    s["out"] = torch.where(live[:, :, None, None], o, s["out"])


def run(s):
    c = s["case"]
    if c["kind"] == "attend8":
        if own:
            from paper_2609_09338_gb300 import binding as ob
            ob.osprey_kv8_attend(s["ctx"], s["kv"], 0, s["n_rows"], s["q"], s["out"], s["status"],
                                 rotate=c["rotate"], advanced=c["advanced"])
        else:
            _plain_attend(s)
        return s["out"]
    if c["advance"]:
        s["seq_len"].copy_(s["start"])   # the batch begins again
    layer = None if c["advance"] else 0
    if own:
        from paper_2609_09338_gb300 import binding as ob
        call = ob.osprey_kv_append_rope if c["kind"] == "append" else ob.osprey_kv8_append
        call(s["ctx"], s["kv"], s["n_rows"], s["k_rows"], s["v_rows"], s["status"], layer=layer, advance=c["advance"])
    else:
        (_plain_append if c["kind"] == "append" else _plain_append8)(s)
        if c["advance"]:
            s["seq_len"] += s["n_rows"]
    if c["kind"] == "append":
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "seq_len": s["seq_len"]}
    # codes as the numbers that they stand for, in units of their block's scale
    return {"k": s["k8"].view(FP8), "v": s["v8"].view(FP8), "k_scale": s["k_scale"], "v_scale": s["v_scale"],
            "k_tail": s["k_tail"], "v_tail": s["v_tail"], "seq_len": s["seq_len"]}


# ---------------------------------------------------------------- work
def work(case):
    """Bytes and operations of one pass, for the mean numbers of rows and lengths."""
    B, Hq, Hkv, hd = case["B"], case["Hq"], case["Hkv"], case["hd"]
    elem = 4 if case["dtype"] == "f32" else 2
    rows = (case["rows_lo"] + case["rows_hi"]) / 2
    if case["kind"] == "attend8":
        ctx = (case["ctx_lo"] + case["ctx_hi"]) / 2
        cache = Hkv * (2 * hd * ctx + 8 * ctx / PAGE)
        return {"bytes": B * (cache + 2 * rows * Hq * hd * elem), "flops": 4.0 * B * Hq * hd * rows * max(1, ctx - rows / 2)}
    layers = case["L"] if case["advance"] else 1
    total = max(1.0, B * rows) * layers * Hkv * hd * 2
    if case["kind"] == "append":
        moved = total * (elem + 2)
    elif case["advance"]:    # a prompt: nearly all of it ends in 8 bits
        moved = total * (elem + 1)
    else:                    # a few rows: into the tail, and a sixteenth of them finishes a page
        moved = total * (elem + 2 + 2 + 1)
    return {"bytes": moved, "flops": 3.0 * total / 2}


# ---------------------------------------------------------------- 64 bits
def _exact_turn(x, pos):
    """x [heads, hd] of one row, float64, turned to its position as complex numbers."""
    h = x.shape[-1] // 2
    freq = THETA ** (-torch.arange(h, device=DEV, dtype=F64) / h)
    z = torch.complex(x[..., :h], x[..., h:]) * torch.polar(torch.ones(h, dtype=F64, device=DEV), pos * freq)
    return torch.cat([z.real, z.imag], -1)


def _exact_blocks(x, values):
    """Codes of blocks [n, Hkv, 16, hd] (float64 holding bf16 values) by the nearest entry of the table of all codes."""
    table = torch.arange(128, dtype=torch.uint8, device=DEV).view(FP8).to(F64)[:127]     # 0 .. 448 ascending
    peak = x.abs().amax((-2, -1))
    e = torch.ceil(torch.log2(torch.clamp(peak, min=1e-300) / 448)).clamp_min(-100)
    e = torch.where(peak > 448 * torch.exp2(e), e + 1, e)
    e = torch.where(peak <= 448 * torch.exp2(e - 1), e - 1, e).clamp_min(-100)
    scale = torch.exp2(e)
    y = x.abs() / scale[..., None, None]
    hi = torch.searchsorted(table, y.contiguous()).clamp(1, 126)
    up, down = table[hi] - y, y - table[hi - 1]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)          # ties to the even code
    y = table[pick] * torch.sign(x)
    n, H, P, hd = x.shape
    if values:
        y = y.permute(0, 1, 3, 2)
    else:
        y = torch.stack([torch.cat([y[:, :, g:g + 8, d:d + 16] for d in range(0, hd, 16)], 2) for g in (0, 8)], 2)
    return y.reshape(n, H, P * hd), scale


def exact(case, seed):
    s = prepare(case, seed)
    B, Hkv, hd, T = case["B"], case["Hkv"], case["hd"], s["tail"]
    G = case["Hq"] // Hkv
    if case["kind"] == "attend8":
        out = s["out"].to(F64)
        for b, (n, total) in enumerate(zip(s["n_host"], s["lens_host"])):
            if not n:
                continue
            full = total // PAGE
            ids = s["table"][b, :full].to(torch.int64)
            keys, vals = [], []
            if full:
                k = s["k8"][0, ids].view(FP8).to(F64).reshape(full, Hkv, 2, hd // 16, 8, 16)
                k = k.permute(0, 2, 4, 1, 3, 5).reshape(full, PAGE, Hkv, hd) * s["k_scale"][0, ids].to(F64)[:, None, :, None]
                v = s["v8"][0, ids].view(FP8).to(F64).reshape(full, Hkv, hd, PAGE)
                v = v.permute(0, 3, 1, 2) * s["v_scale"][0, ids].to(F64)[:, None, :, None]
                keys.append(k.reshape(-1, Hkv, hd))
                vals.append(v.reshape(-1, Hkv, hd))
            at = b * T + full % T
            rest = total - full * PAGE
            keys.append(s["k_tail"][0, at, :, :rest].to(F64).transpose(0, 1))
            vals.append(s["v_tail"][0, at, :, :rest].to(F64).transpose(0, 1))
            k, v = torch.cat(keys), torch.cat(vals)
            pos = torch.arange(total - n, total, device=DEV)
            q = s["q"][b, :n].to(F64)
            if case["rotate"]:
                q = torch.stack([_exact_turn(x, float(total - n + j)) for j, x in enumerate(q)])
            hidden = torch.arange(total, device=DEV)[None] > pos[:, None]
            for h in range(Hkv):
                z = q[:, h * G:(h + 1) * G].reshape(n * G, hd) @ k[:, h].T / hd ** 0.5
                z = z.masked_fill(hidden.repeat_interleave(G, 0), -math.inf)
                z = torch.softmax(z, -1)
                out[b, :n, h * G:(h + 1) * G] = (z @ v[:, h]).reshape(n, G, hd)
        return out
    kr, vr = (s["k_rows"], s["v_rows"]) if case["advance"] else (s["k_rows"][None], s["v_rows"][None])
    L = kr.shape[0]
    seqs = [(b, st, n) for b, (st, n) in enumerate(zip(s["lens_host"], s["n_host"]))]
    pos = torch.cat([torch.arange(st, st + n, device=DEV, dtype=F64) for _, st, n in seqs])
    h = hd // 2
    turn = torch.polar(torch.ones((len(pos), h), dtype=F64, device=DEV),
                       pos[:, None] * THETA ** (-torch.arange(h, device=DEV, dtype=F64) / h))[:, None]
    z = torch.complex(kr[..., :h].to(F64), kr[..., h:].to(F64)) * turn
    k = torch.cat([z.real, z.imag], -1).to(BF)
    v = vr.to(BF)
    seq_len = s["start"] + (s["n_rows"] if case["advance"] else 0)
    if case["kind"] == "append":
        kp, vp = s["k_pages"].clone(), s["v_pages"].clone()
        r = 0
        for b, st, n in seqs:
            at = torch.arange(st, st + n, device=DEV)
            ids = s["table"][b, at // PAGE].to(torch.int64)
            for layer in range(L):
                kp[layer, ids, :, at % PAGE] = k[layer, r:r + n]
                vp[layer, ids, :, at % PAGE] = v[layer, r:r + n]
            r += n
        return {"k_pages": kp.to(F64) if kp.numel() < 1e8 else kp, "v_pages": vp, "seq_len": seq_len}
    got = {"k": s["k8"].view(FP8).to(F32), "v": s["v8"].view(FP8).to(F32), "k_scale": s["k_scale"].to(F64),
           "v_scale": s["v_scale"].to(F64), "k_tail": s["k_tail"].to(F64), "v_tail": s["v_tail"].to(F64),
           "seq_len": seq_len}
    for name, new in (("k", k), ("v", v)):
        r = 0
        for b, st, n in seqs:
            if not n:
                continue
            p0, p1 = st // PAGE, (st + n - 1) // PAGE
            # the rows of the pages touched, laid one after another behind the older rows of the first one
            older = s[name + "_tail"][:L, b * T + p0 % T, :, :st - p0 * PAGE].transpose(1, 2)
            rows = torch.cat([older, new[:, r:r + n]], 1).to(F64)                       # [L, rows, Hkv, hd]
            r += n
            full = rows.shape[1] // PAGE
            if full:
                ids = s["table"][b, p0:p0 + full].to(torch.int64)
                for layer in range(L):
                    x = rows[layer, :full * PAGE].reshape(full, PAGE, Hkv, hd).transpose(1, 2)
                    code, scale = _exact_blocks(x, name == "v")
                    got[name][layer, ids] = code.to(F32)
                    got[name + "_scale"][layer, ids] = scale
            for p in range(max(p0, p1 - T + 1), p1 + 1):
                lo, hi = max(st, p * PAGE), min(st + n, (p + 1) * PAGE)
                x = rows[:, lo - p0 * PAGE:hi - p0 * PAGE].transpose(1, 2)
                got[name + "_tail"][:L, b * T + p % T, :, lo - p * PAGE:hi - p * PAGE] = x
    return got
