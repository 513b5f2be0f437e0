"""The operators around a proposal or verification step whose speed is measured:
appending rotated keys and values to the paged cache, attention of sequences
that share a prefix, and drawing a token from filtered logits.

Each has a plain form in elementary torch operations (``own`` false) and the
library's call (``own`` true), marshalled once and reissued, as the executor
does. A case is a dict of plain values; sizes follow from the case alone,
values from the seed.

* ``rope``: tokens of a fused projection [T][(Hq + 2 Hkv) D] are rotated by
  their positions (one to three axes) and K and V written into their pages.
* ``shared``: groups of sequences with common leading pages; windows of one
  token (a decode step) and more.
* ``sample``: temperature, top-k, top-p and min-p, one uniform number a row.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda"
ELEM = {"f32": 4, "bf16": 2, "fp8": 1}
POOL = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}
F8 = torch.float8_e4m3fn


def _rope(name, seqs, new, kv, *, hq=32, hkv=8, dim=128, rot=128, axes=1, halves=True, aligned=True):
    c = {"op": "rope", "seqs": seqs, "new": new, "kv": kv, "hq": hq, "hkv": hkv, "dim": dim,
         "rot": rot, "axes": axes, "halves": halves, "aligned": aligned}
    return {"name": name, **c} if name else c


def _shared(name, groups, size, prefix, own_tokens, kv, *, hq=32, hkv=8, dim=128, window=1,
            ragged=False):
    c = {"op": "shared", "groups": groups, "size": size, "prefix": prefix, "own": own_tokens,
         "kv": kv, "hq": hq, "hkv": hkv, "dim": dim, "window": window, "ragged": ragged}
    return {"name": name, **c} if name else c


def _sample(name, rows, vocab, logits, mode):
    c = {"op": "sample", "rows": rows, "vocab": vocab, "logits": logits, "mode": mode}
    return {"name": name, **c} if name else c


def listed():
    return [
        # The next token of one sequence: launch latency.
        _rope("rope_1", 1, 1, "bf16"),
        # The 5-token windows of a 64-sequence serving batch, fp8 pages.
        _rope("rope_64x5_fp8", 64, 5, "fp8", aligned=False),
        # A chunked-prefill step of a vision-language model: four requests'
        # next 2048 tokens, positions along time, height and width.
        _rope("rope_prefill", 4, 2048, "bf16", axes=3),
        # Reference serving in float32: a ragged chunk, half of each head
        # rotated, neighbouring dims paired, 64-dim heads.
        _rope("rope_f32_partial", 3, 1237, "f32", hq=16, hkv=8, dim=64, rot=32, halves=False,
              aligned=False),
        # A decode step of eight questions about one 16K document.
        _shared("shared_8x16k", 1, 8, 16384, 256, "bf16"),
        # The same of 64 questions about a 32K document: as much arithmetic as bytes.
        _shared("shared_64x32k", 1, 64, 32768, 512, "bf16", ragged=True),
        # Four documents of up to 128K with four questions each, 5-token windows, fp8 pages.
        _shared("shared_verify_fp8", 4, 4, 131072, 1024, "fp8", window=5, ragged=True),
        # Reference serving in float32: two short sequences with 64-dim heads.
        _shared("shared_2_f32", 1, 2, 1000, 40, "f32", hq=16, hkv=8, dim=64),
        # The next token of one sequence, a small vocabulary, in float32.
        _sample("sample_1", 1, 32000, "f32", "mixed"),
        # The proposal step of a 64-sequence batch, parameters of their own each.
        _sample("sample_64", 64, 151936, "bf16", "mixed"),
        # Every position of 64 five-token windows, nucleus only, an odd vocabulary.
        _sample("sample_320_top_p", 320, 151937, "bf16", "top_p"),
        # Drawing from the whole distribution, float32 logits.
        _sample("sample_16_f32", 16, 128000, "f32", "all"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["rope", "shared", "sample"], [3, 4, 3])[0]
    if op == "sample":
        vocab = _log(rng, 1000, 200000)
        rows = min(_log(rng, 1, 320), (320 * 151936) // vocab)
        return _sample(None, rows, vocab, rng.choice(["bf16", "f32"]),
                       rng.choice(["mixed", "mixed", "top_k", "top_p", "all"]))
    kv = rng.choice(["bf16", "bf16", "fp8", "f32"])
    if rng.random() < 0.5:
        hkv, group, dim = rng.choice([2, 4, 8]), 4, 128
    else:
        hkv, group, dim = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 6, 8]), \
            rng.choice([64, 128, 256])
    hq = hkv * group
    if op == "rope":
        es = 4 if kv == "f32" else 2
        new = _log(rng, 1, 4096)
        seqs = max(1, min(_log(rng, 1, 64), (96 << 20) // (new * (hq + 2 * hkv) * dim * es)))
        rot = rng.choice([dim, dim, dim // 2, 48])
        return _rope(None, seqs, new, kv, hq=hq, hkv=hkv, dim=dim, rot=rot,
                     axes=rng.choice([1, 2, 3]), halves=rng.random() < 0.7,
                     aligned=rng.random() < 0.5)
    size, groups = _log(rng, 2, 64), rng.choice([1, 1, 2, 4])
    window = rng.choice([1, 1, 1, 3, 5, 8])
    prefix = _log(rng, 256, 131072 if kv != "f32" else 16384)
    most = (512 << 20) if kv != "f32" else (128 << 20)
    prefix = max(32, min(prefix, most // (groups * 2 * hkv * dim * ELEM[kv])))
    own_tokens = min(_log(rng, 16, 2048), max(16, prefix // 2))
    own_tokens = max(16, min(own_tokens, most // (groups * size * 2 * hkv * dim * ELEM[kv])))
    # (at most the arithmetic of 2048 query rows over 32K keys of 128 dims)
    rows = hq * size * window * groups
    prefix = max(32, min(prefix, (4 << 30) // (rows * dim // 2)))
    return _shared(None, groups, size, prefix, max(own_tokens, window), kv, hq=hq, hkv=hkv,
                   dim=dim, window=window, ragged=rng.random() < 0.5)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) % (1 << 62))


def _dev(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x)).to(dtype).to(DEV)


def _pool(c, pages, gen):
    """K and V pools, iid N(0, 1); fp8: codes and a scale per page."""
    kv, hkv, dim = c["kv"], c["hkv"], c["dim"]
    pools, scales = [], torch.empty((pages, 2), dtype=torch.float32, device=DEV) \
        if kv == "fp8" else None
    for i, shape in enumerate(((pages, hkv, dim // 8, PAGE, 8), (pages, hkv, dim, PAGE))):
        dst = torch.empty(shape, dtype=POOL[kv], device=DEV)
        step = max(1, (256 << 20) // (hkv * dim * PAGE * 4))
        for p in range(0, pages, step):
            if kv != "fp8":
                dst[p:p + step].normal_(generator=gen)
                continue
            x = torch.randn(dst[p:p + step].shape, generator=gen, device=DEV)
            s = x.abs().flatten(1).amax(1) / 448.0
            scales[p:p + step, i] = s
            x = (x / s.view(-1, *[1] * (x.dim() - 1))).clamp_(-448.0, 448.0)
            dst[p:p + step].copy_(x.to(F8).view(torch.uint8))
        pools.append(dst)
    return pools[0], pools[1], scales


def _prepare_rope(c, seed):
    r, gen = np.random.default_rng(seed), _gen(seed)
    seqs, new, hq, hkv, dim, rot = (c[k] for k in ("seqs", "new", "hq", "hkv", "dim", "rot"))
    T = seqs * new
    # pages of the new tokens: each sequence's own, in shuffled order, starting inside one
    start = np.zeros(seqs, np.int64) if c["aligned"] else r.integers(0, PAGE, seqs)
    per = -(-(int(start.max()) + new) // PAGE)
    pages = r.permutation(seqs * per).reshape(seqs, per)
    off = start[:, None] + np.arange(new)[None, :]
    slots = (np.take_along_axis(pages, off // PAGE, 1) * PAGE + off % PAGE).reshape(-1)
    if T > 16:
        slots[r.integers(0, T, max(1, T // 64))] = -1            # padding of a fixed-size step
    first = PAGE * r.integers(0, 4096, seqs) + start             # position of the first new token
    t = first[:, None] + np.arange(new)[None, :]
    wide = int(r.integers(8, 48))                                # patches in a row of an image
    grid = np.arange(new)[None, :] + 0 * first[:, None]
    axes = [t, first[:, None] + grid // wide, first[:, None] + grid % wide]
    if c["axes"] > 1:
        axes[0] = first[:, None] + grid // 256
    positions = np.stack([a.reshape(-1) for a in axes[:c["axes"]]])
    inv = (1e6 ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)
    k_pages, v_pages, scales = _pool(c, seqs * per, gen)
    dt = torch.float32 if c["kv"] == "f32" else torch.bfloat16
    qkv = torch.randn((T, (hq + 2 * hkv) * dim), generator=gen, device=DEV).to(dt)
    q, k, v = qkv.split([hq * dim, hkv * dim, hkv * dim], 1)
    s = {"c": c, "q": q.view(T, hq, dim), "k": k.view(T, hkv, dim), "v": v.view(T, hkv, dim),
         "slots": _dev(slots, torch.int64), "positions": _dev(positions),
         "inv_freq": _dev(inv, torch.float32), "freq_axis": _dev(np.arange(rot // 2) % c["axes"]),
         "k_pages": k_pages, "v_pages": v_pages, "scales": scales,
         "q_out": torch.empty((T, hq, dim), dtype=dt, device=DEV)}
    if own:
        from paper_2607_24260_amd import kap as K
        kv = K.KVCache(k_pages, v_pages, hq, dt, scales)
        style = K.KAP_ROPE_HALVES if c["halves"] else K.KAP_ROPE_PAIRS
        s["call"] = K.bind_rope_append_kv(kv, s["k"], s["v"], s["slots"], s["positions"],
                                          s["inv_freq"], q_new=s["q"], q_out=s["q_out"],
                                          freq_axis=s["freq_axis"], style=style)
    return s


def _shared_sizes(c):
    """(shared pages per group, sequence lengths [groups][size]) from the case alone."""
    n, m = c["groups"], c["size"]
    blocks = np.full(n, -(-c["prefix"] // PAGE), np.int64)
    tokens = np.full((n, m), c["own"], np.int64)
    if c["ragged"]:
        r = np.random.default_rng(c["prefix"] * 131 + n * m)
        blocks[1:] = np.maximum(1, (blocks[1:] * r.uniform(0.25, 1.0, n - 1)).astype(np.int64))
        tokens = np.maximum(c["window"], (tokens * r.uniform(0.1, 1.0, (n, m))).astype(np.int64))
    return blocks, blocks[:, None] * PAGE + tokens


def _prepare_shared(c, seed):
    r, gen = np.random.default_rng(seed), _gen(seed)
    n, m, hq, dim, w = (c[k] for k in ("groups", "size", "hq", "dim", "window"))
    blocks, lens = _shared_sizes(c)
    pages = -(-lens // PAGE)
    total = int(blocks.sum() + (pages - blocks[:, None]).sum())
    perm, at = r.permutation(total), 0
    table = np.zeros((n, m, int(pages.max())), np.int64)
    for g in range(n):
        table[g, :, :blocks[g]] = perm[at:at + blocks[g]]
        at += int(blocks[g])
        for i in range(m):
            k = int(pages[g, i] - blocks[g])
            table[g, i, blocks[g]:pages[g, i]] = perm[at:at + k]
            at += k
    k_pages, v_pages, scales = _pool(c, total, gen)
    dt = torch.float32 if c["kv"] == "f32" else torch.bfloat16
    B = n * m
    s = {"c": c, "k_pages": k_pages, "v_pages": v_pages, "scales": scales,
         "q": torch.randn((B, w, hq, dim), generator=gen, device=DEV).to(dt),
         "lens": _dev(lens.reshape(-1)), "table": _dev(table.reshape(B, -1)),
         "offsets": _dev(np.arange(n + 1) * m), "blocks": _dev(blocks),
         "most": int(lens.max()), "scale": 1.0 / math.sqrt(dim),
         "prefix_pages": int(blocks.max()), "own_pages": int((pages - blocks[:, None]).max()),
         "out": torch.empty((B, w, hq, dim), dtype=torch.float32, device=DEV),
         "lse": torch.empty((B, w, hq), dtype=torch.float32, device=DEV)}
    if own:
        from paper_2607_24260_amd import kap as K
        kv = K.KVCache(k_pages, v_pages, hq, dt, scales)
        ws = torch.zeros(max(256, K.verify_shared_workspace_bytes(kv, B, w, s["most"], n)),
                         dtype=torch.uint8, device=DEV)
        s["call"] = K.bind_verify_shared(kv, s["q"], s["lens"], s["table"], s["most"],
                                         s["offsets"], s["blocks"], s["scale"], s["out"],
                                         s["lse"], ws)
    return s


def _prepare_sample(c, seed):
    r, gen = np.random.default_rng(seed), _gen(seed)
    rows, vocab = c["rows"], c["vocab"]
    x = torch.randn((rows, vocab), generator=gen, device=DEV) * 2.5
    # a few likely tokens in every row, as a trained model's logits have
    at = torch.randint(0, vocab, (rows, 12), generator=gen, device=DEV)
    x.scatter_add_(1, at, torch.rand((rows, 12), generator=gen, device=DEV) * 14)
    x = x.to(torch.float32 if c["logits"] == "f32" else torch.bfloat16)
    mode = c["mode"]
    temp = r.uniform(0.5, 1.3, rows)
    top_k = np.zeros(rows, np.int64)
    top_p, min_p = np.ones(rows), np.zeros(rows)
    if mode in ("mixed", "top_k"):
        top_k = r.choice([1, 20, 40, 50, 200], rows)
    if mode in ("mixed", "top_p"):
        top_p = r.choice([0.8, 0.9, 0.95, 0.98], rows)
    if mode == "mixed":
        temp[r.random(rows) < 0.1] = 0.0                         # greedy rows
        top_k[r.random(rows) < 0.5] = 0                          # and rows without a top-k,
        top_p[r.random(rows) < 0.4] = 1.0                        # a top-p,
        min_p = np.where(r.random(rows) < 0.5, 0.0, r.choice([0.02, 0.05, 0.1], rows))
    f32 = torch.float32
    s = {"c": c, "logits": x, "temperature": _dev(temp, f32), "top_k": _dev(top_k),
         "top_p": _dev(top_p, f32), "min_p": _dev(min_p, f32),
         "uniform": torch.rand(rows, generator=gen, device=DEV),
         "token": torch.empty(rows, dtype=torch.int32, device=DEV),
         "prob": torch.empty(rows, dtype=f32, device=DEV)}
    if own:
        from paper_2607_24260_amd import kap as K
        ws = torch.zeros(max(256, K.sample_workspace_bytes(rows, vocab)), dtype=torch.uint8,
                         device=DEV)
        s["call"] = K.bind_sample(x, s["uniform"], temperature=s["temperature"],
                                  top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"],
                                  token=s["token"], prob=s["prob"], workspace=ws)
    return s


def prepare(case, seed):
    return {"rope": _prepare_rope, "shared": _prepare_shared,
            "sample": _prepare_sample}[case["op"]](case, seed)


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def _rotate(x, cos, sin, rot, halves):
    """x [T][H][D] float32 with the pairs of its first ``rot`` dims turned."""
    y, h = x.clone(), rot // 2
    a, b = (slice(0, h), slice(h, rot)) if halves else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _rope_plain(s):
    c = s["c"]
    pos = s["positions"][s["freq_axis"].long()].double().T       # [T][rot/2]
    angle = pos * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    q = _rotate(s["q"].float(), cos, sin, c["rot"], c["halves"])
    k = _rotate(s["k"].float(), cos, sin, c["rot"], c["halves"])
    v = s["v"].float()
    live = (s["slots"] >= 0).nonzero().squeeze(1)
    page, off = s["slots"][live] // PAGE, s["slots"][live] % PAGE
    k, v = k[live], v[live]
    if c["kv"] == "fp8":
        store = lambda x, i: (x / s["scales"][page, i].view(-1, 1, 1)).clamp(
            -448.0, 448.0).to(F8).view(torch.uint8)
    else:
        store = lambda x, i: x.to(s["k_pages"].dtype)
    s["k_pages"][page, :, :, off] = store(k, 0).unflatten(2, (c["dim"] // 8, 8))
    s["v_pages"][page, :, :, off] = store(v, 1)
    s["q_out"].copy_(q)


def _values(pages, scales, i, dtype):
    """A gathered run of pages [..., n, ...] as numbers."""
    x = pages.view(F8).to(dtype) if pages.dtype == torch.uint8 else pages.to(dtype)
    return x if scales is None else x * scales[..., i].to(dtype).view(
        *scales.shape[:-1], *[1] * (x.dim() - scales.dim() + 1))


def _keys(s, table, dtype):
    """K and V [rows][Hkv][tokens][D] of the pages in a table [rows][pages]."""
    n, p = table.shape
    dim, hkv = s["c"]["dim"], s["c"]["hkv"]
    sc = None if s["scales"] is None else s["scales"][table]
    k = _values(s["k_pages"][table], sc, 0, dtype)               # [n][p][Hkv][D/8][16][8]
    v = _values(s["v_pages"][table], sc, 1, dtype)               # [n][p][Hkv][D][16]
    k = k.permute(0, 2, 1, 4, 3, 5).reshape(n, hkv, p * PAGE, dim)
    v = v.permute(0, 2, 1, 4, 3).reshape(n, hkv, p * PAGE, dim)
    return k, v


def _shared_plain(s, dtype=torch.float32):
    """Attention with the prefixes read once: logits of the groups' shared pages
    and of each sequence's own ones side by side."""
    c = s["c"]
    n, m, w, hq, hkv, dim = (c[k] for k in ("groups", "size", "window", "hq", "hkv", "dim"))
    B, G, P = n * m, hq // hkv, s["prefix_pages"]
    table, lens, blocks = s["table"].long(), s["lens"].long(), s["blocks"].long()
    own_at = (blocks.repeat_interleave(m)[:, None] + torch.arange(s["own_pages"], device=DEV))
    own_table = table.gather(1, own_at.clamp(max=table.shape[1] - 1))
    kp, vp = _keys(s, table.view(n, m, -1)[:, 0, :P], dtype)     # the groups' shared pages
    ko, vo = _keys(s, own_table, dtype)
    q = s["q"].to(dtype).view(n, m, w, hkv, G, dim).permute(0, 3, 1, 2, 4, 5)
    zp = torch.matmul(q.reshape(n, hkv, m * w * G, dim), kp.transpose(2, 3))
    qo = q.permute(0, 2, 1, 3, 4, 5).reshape(B, hkv, w * G, dim)
    zo = torch.matmul(qo, ko.transpose(2, 3))                    # [B][Hkv][w G][own tokens]
    z = torch.cat([zp.view(n, hkv, m, w * G, -1).transpose(1, 2).reshape(B, hkv, w * G, -1), zo],
                  -1) * s["scale"]
    # positions of the keys, and the last one each row sees
    at = torch.cat([torch.arange(P * PAGE, device=DEV).expand(B, -1),
                    (own_at[:, :, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten(1)], 1)
    shared = (blocks * PAGE).repeat_interleave(m)[:, None]
    real = torch.ones_like(at, dtype=torch.bool)
    real[:, :P * PAGE] = at[:, :P * PAGE] < shared
    last = lens[:, None] - w + torch.arange(w, device=DEV)       # [B][w]
    seen = real[:, None] & (at[:, None] <= last[:, :, None])     # [B][w][tokens]
    z = z.view(B, hkv, w, G, -1).masked_fill(~seen[:, None, :, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(-1, keepdim=True)
    e = (e / total).view(B, hkv, w * G, -1)
    ep = e[..., :P * PAGE].view(n, m, hkv, w * G, -1).transpose(1, 2).reshape(n, hkv, m * w * G, -1)
    o = torch.matmul(ep, vp).view(n, hkv, m, w * G, dim).transpose(1, 2).reshape(B, hkv, w * G, dim)
    o = o + torch.matmul(e[..., P * PAGE:], vo)
    out = o.view(B, hkv, w, G, dim).transpose(1, 2).reshape(B, w, hq, dim)
    lse = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(B, w, hq)
    return out, lse


def _sample_plain(s):
    x = s["logits"].double()
    vocab = x.shape[1]
    x, index = x.sort(dim=1, descending=True, stable=True)         # ties: the lowest index first
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    e = ((x - x[:, :1]) / torch.where(greedy, 1.0, t)).exp()
    sums = e.cumsum(1)
    k = s["top_k"].long()[:, None]
    k = torch.where((k <= 0) | (k > vocab), vocab, k)
    p = s["top_p"].double()[:, None]
    in_k = sums.gather(1, k - 1)
    r_p = torch.where(p >= 1, vocab, (sums < p * in_k).sum(1, keepdim=True) + 1)
    r_m = (e >= s["min_p"].double()[:, None]).sum(1, keepdim=True)
    kept = torch.minimum(torch.minimum(k, r_p), r_m)
    kept = torch.where(greedy, 1, kept).clamp(min=1)
    total = sums.gather(1, kept - 1)
    u = s["uniform"].double()[:, None]
    rank = torch.minimum((sums <= u * total).sum(1, keepdim=True), kept - 1)
    s["token"].copy_(index.gather(1, rank).squeeze(1))
    s["prob"].copy_((e.gather(1, rank) / total).squeeze(1))


def run(state):
    s, op = state, state["c"]["op"]
    if op == "rope":
        s["call"]() if own else _rope_plain(s)
        if s["c"]["kv"] == "fp8":
            return [s["q_out"], s["k_pages"].view(F8), s["v_pages"].view(F8)]
        return [s["q_out"], s["k_pages"], s["v_pages"]]
    if op == "shared":
        if not own:
            return list(_shared_plain(s))
        s["call"]()
        return [s["out"], s["lse"]]
    s["call"]() if own else _sample_plain(s)
    return [s["token"], s["prob"]]


def work(case):
    c = case
    if c["op"] == "sample":
        n = c["rows"] * c["vocab"]
        # a maximum, an exponential and a sum for each logit
        return {"bytes": n * (4 if c["logits"] == "f32" else 2) + c["rows"] * 28, "flops": 4 * n}
    es, ek = (4 if c["kv"] == "f32" else 2), ELEM[c["kv"]]
    if c["op"] == "rope":
        T, d = c["seqs"] * c["new"], c["dim"]
        return {"bytes": T * ((2 * c["hq"] + 2 * c["hkv"]) * d * es + 2 * c["hkv"] * d * ek
                              + 8 + 4 * c["axes"]),
                "flops": 3 * T * (c["hq"] + c["hkv"]) * c["rot"]}
    blocks, lens = _shared_sizes(c)
    tokens = int(blocks.sum()) * PAGE + int((lens - blocks[:, None] * PAGE).sum())
    w, hq, d = c["window"], c["hq"], c["dim"]
    rows = c["groups"] * c["size"] * w * hq
    seen = int(lens.sum()) * w - c["groups"] * c["size"] * w * (w - 1) // 2
    return {"bytes": tokens * 2 * c["hkv"] * d * ek + rows * (d * (es + 4) + 4),
            "flops": 4 * d * hq * seen}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------

def _exact_rope(c, s):
    f = lambda x: x.double().cpu().numpy()
    pos, axis = s["positions"].cpu().numpy().astype(np.float64), s["freq_axis"].cpu().numpy()
    turn = np.exp(1j * (pos[axis].T * f(s["inv_freq"])))[:, None, :]

    def rotated(x):
        h = c["rot"] // 2
        y = x.copy()
        if c["halves"]:
            z = (x[..., :h] + 1j * x[..., h:2 * h]) * turn
            y[..., :h], y[..., h:2 * h] = z.real, z.imag
        else:
            z = (x[..., 0:2 * h:2] + 1j * x[..., 1:2 * h:2]) * turn
            y[..., 0:2 * h:2], y[..., 1:2 * h:2] = z.real, z.imag
        return y

    def pool(x):
        return f(x.view(F8) if x.dtype == torch.uint8 else x)

    k, v = rotated(f(s["k"])), f(s["v"])
    kp, vp = pool(s["k_pages"]), pool(s["v_pages"])
    slots = s["slots"].cpu().numpy()
    live = np.nonzero(slots >= 0)[0]
    page, off = slots[live] // PAGE, slots[live] % PAGE
    k, v = k[live], v[live]
    if c["kv"] == "fp8":
        sc = f(s["scales"])[page]
        k = np.clip(k / sc[:, 0, None, None], -448, 448)
        v = np.clip(v / sc[:, 1, None, None], -448, 448)
    kp[page, :, :, off] = k.reshape(len(live), c["hkv"], c["dim"] // 8, 8)
    vp[page, :, :, off] = v
    return [rotated(f(s["q"])), kp, vp]


def _exact_shared(c, s):
    """Each sequence by itself over its whole table, no use made of what is shared."""
    hkv, G, w, dim = c["hkv"], c["hq"] // c["hkv"], c["window"], c["dim"]
    outs, lses = [], []
    for b in range(c["groups"] * c["size"]):
        L = int(s["lens"][b])
        pages = s["table"][b, :-(-L // PAGE)].long()
        k = s["k_pages"][pages]
        v = s["v_pages"][pages]
        if c["kv"] == "fp8":
            k = k.view(F8).double() * s["scales"][pages, 0].double().view(-1, 1, 1, 1, 1)
            v = v.view(F8).double() * s["scales"][pages, 1].double().view(-1, 1, 1, 1)
        k = k.double().transpose(2, 3).flatten(3).transpose(0, 1).flatten(1, 2)[:, :L]
        v = v.double().transpose(2, 3).transpose(0, 1).flatten(1, 2)[:, :L]
        q = s["q"][b].double().view(w, hkv, G, dim).transpose(0, 1)      # [Hkv][w][G][D]
        z = torch.matmul(q.reshape(hkv, w * G, dim), k.transpose(1, 2).contiguous()) * s["scale"]
        z = z.view(hkv, w, G, L)
        hidden = torch.arange(L, device=DEV)[None, :] > L - w + torch.arange(w, device=DEV)[:, None]
        z = z.masked_fill(hidden[None, :, None], -math.inf)
        lse = torch.logsumexp(z, -1)
        o = torch.matmul((z - lse[..., None]).exp().view(hkv, w * G, L), v)
        outs.append(o.view(hkv, w, G, dim).transpose(0, 1).reshape(w, hkv * G, dim))
        lses.append(lse.transpose(0, 1).reshape(w, hkv * G))
    return [torch.stack(outs), torch.stack(lses)]


def _exact_sample(c, s):
    x = s["logits"].float().cpu().numpy().astype(np.float64)
    par = {k: s[k].cpu().numpy().astype(np.float64)
           for k in ("temperature", "top_k", "top_p", "min_p", "uniform")}
    tokens, probs = [], []
    for i in range(c["rows"]):
        order = np.argsort(-x[i], kind="stable")
        if par["temperature"][i] <= 0:
            tokens.append(order[0])
            probs.append(1.0)
            continue
        e = np.exp((x[i, order] - x[i, order[0]]) / par["temperature"][i])
        k = int(par["top_k"][i])
        k = k if 0 < k < len(e) else len(e)
        n = k
        if par["top_p"][i] < 1:
            n = min(n, int(np.searchsorted(np.cumsum(e[:k]), par["top_p"][i] * e[:k].sum())) + 1)
        n = max(1, min(n, int((e >= par["min_p"][i]).sum())))
        sums = np.cumsum(e[:n])
        r = min(int(np.searchsorted(sums, par["uniform"][i] * sums[-1], side="right")), n - 1)
        tokens.append(order[r])
        probs.append(e[r] / sums[-1])
    return [np.asarray(tokens, np.int32), np.asarray(probs)]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    return {"rope": _exact_rope, "shared": _exact_shared, "sample": _exact_sample}[c["op"]](c, s)
