"""kap_chunk_attention against attention in 64 bits.

Bounds. A logit is a sum of D exact products (of bf16 values; float32 ones are rounded)
in single precision: off by at most z = (D + 4) 2^-24 scale |q| |k|. The lse is then off by
z and a few roundings, and so is each weight, relative to it, on top of the rounding of
its sum over n keys: n 2^-24 at most, and of the exponential. An output is a mean of V
with those weights: off by A (2 z + n 2^-24 + 2^-20) with A the mean of |V|. With bf16 and fp8
pages each weight is rounded to bf16, and so is the output: 2^-8 (A + |o|) more.
Weights below 2^-126 come out as 0, against a largest one of 2^-8 at least (the
reference is up to 8 above the largest logit): n times 2^-118 |v| in an output, |v| < 8 here.
"""
import math

import numpy as np
import pytest
import torch

from oracle import kap_oracle as O
from paper_2607_24260_amd import kap as K
from paper_2607_24260_amd.workloads import kv_pool

from kap_testlib import dev_i32, server_batch

pytestmark = pytest.mark.gpu

QDT = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
FILL = 7.0


class Chunks:
    """Sequences of (new tokens, length); ``pad`` rows behind the last."""

    def __init__(self, dtype, seqs, *, Hq=8, Hkv=2, D=128, window=0, sinks=0, seed=1, pad=3, wide=0,
                 spread=1.0, scale=None):
        rng = np.random.default_rng(seed)
        self.dtype, self.window, self.sinks, self.D, self.G = dtype, window, sinks, D, Hq // Hkv
        self.new = np.array([n for n, _ in seqs], np.int64)
        self.lens = np.array([L for _, L in seqs], np.int64)
        self.offsets = np.concatenate([[0], np.cumsum(self.new)])
        pages = -(-self.lens.clip(0) // 16)
        total = int(pages.sum()) + 3
        perm, at = rng.permutation(total), 0
        self.table = np.full((len(seqs), max(int(pages.max(initial=0)), 1) + wide), -5)
        for b, p in enumerate(pages):
            self.table[b, :p] = perm[at:at + p]
            at += p
        k, v, sc = kv_pool(total, Hkv, D, dtype, seed + 1, "cuda")
        self.kv = K.KVCache(k, v, Hq, QDT[dtype], sc)
        g = torch.Generator(device="cuda").manual_seed(seed + 2)
        self.T = int(self.offsets[-1]) + pad
        self.q = (torch.randn((self.T, Hq, D), generator=g, device="cuda") * spread).to(QDT[dtype])
        self.scale = 1.0 / math.sqrt(D) if scale is None else scale
        self.most = int(self.lens.max(initial=0))

    def run(self, **kw):
        out = torch.full_like(self.q, FILL)
        lse = torch.full(self.q.shape[:2], FILL, device="cuda")
        K.chunk_attention(self.kv, self.q, dev_i32(self.offsets), dev_i32(self.lens),
                          dev_i32(self.table), max(self.most, 0), self.scale, out=out, lse=lse,
                          window=self.window, sinks=self.sinks, **kw)
        torch.cuda.synchronize()
        return out, lse

    def want(self):
        """(o, lse, A, largest |q| |k|, keys) in 64 bits, with torch on the GPU."""
        kv, D = self.kv, self.D
        T, Hq = self.T, kv.num_q_heads
        o = torch.full((T, Hq, D), FILL, dtype=torch.float64, device="cuda")
        lse = torch.full((T, Hq), FILL, dtype=torch.float64, device="cuda")
        mean, far, most = o.clone(), 0.0, 1
        for b, (n, L) in enumerate(zip(self.new, self.lens)):
            r0 = int(self.offsets[b])
            if n == 0:
                continue
            ids = torch.as_tensor(self.table[b, :-(-max(L, 0) // 16)], device="cuda")
            good = (ids >= 0) & (ids < kv.num_pages)
            at = torch.where(good, ids, 0)
            k, v = kv.k_pages[at], kv.v_pages[at]
            if self.dtype == "fp8":
                f8 = torch.float8_e4m3fn
                k = k.view(f8).double() * kv.kv_scales[at, 0].double().view(-1, 1, 1, 1, 1)
                v = v.view(f8).double() * kv.kv_scales[at, 1].double().view(-1, 1, 1, 1)
            L = max(int(L), 0)
            k = k.double().permute(1, 0, 3, 2, 4).reshape(kv.num_kv_heads, len(ids) * 16, D)[:, :L]
            v = v.double().permute(1, 0, 3, 2).reshape(kv.num_kv_heads, len(ids) * 16, D)[:, :L].contiguous()
            t = torch.arange(L, device="cuda")
            there = good.repeat_interleave(16)[:L]
            for i0 in range(0, n, 512):
                m = min(512, n - i0)
                rows = slice(r0 + i0, r0 + i0 + m)
                p = (L - n + i0 + torch.arange(m, device="cuda"))[:, None]
                seen = (t <= p) & there
                if self.window:
                    seen &= (p - t < self.window) | (t < self.sinks)
                q = self.q[rows].double().view(m, kv.num_kv_heads, self.G, D).transpose(0, 1)
                q = q.reshape(kv.num_kv_heads, m * self.G, D)
                z = torch.matmul(q, k.transpose(1, 2).contiguous()) * self.scale
                z = z.view(kv.num_kv_heads, m, self.G, L).masked_fill(~seen[None, :, None], -math.inf)
                l = torch.logsumexp(z, -1) if L else torch.full(z.shape[:3], -math.inf, device="cuda",
                                                                dtype=torch.float64)
                w = torch.where(seen[None, :, None], (z - l[..., None]).exp(), 0.0)
                w = torch.where(l[..., None] == -math.inf, 0.0, w).view(kv.num_kv_heads, m * self.G, L)
                put = lambda x: x.view(kv.num_kv_heads, m, self.G, D).transpose(0, 1).reshape(m, Hq, D)   # noqa: E731
                o[rows], mean[rows] = put(torch.matmul(w, v)), put(torch.matmul(w, v.abs()))
                lse[rows] = l.transpose(0, 1).reshape(m, Hq)
                if L:
                    far = max(far, float(q.norm(dim=-1).max() * k.norm(dim=-1).max()))
                most = max(most, int(seen.sum(1).max()) if L else 1)
        return o, lse, mean, far, most

    def check(self, **kw):
        out, lse = self.run(**kw)
        o, l, mean, far, most = self.want()
        z = (self.D + 4) * 2.0 ** -24 * abs(self.scale) * far
        tol = mean * (2 * z + most * 2.0 ** -24 + 2.0 ** -20) + most * 8 * 2.0 ** -118
        if self.dtype != "f32":
            tol = tol + 2.0 ** -8 * (mean + o.abs())
        live = slice(0, int(self.offsets[-1]))
        assert bool((out[live.stop:] == FILL).all()) and bool((lse[live.stop:] == FILL).all())
        assert torch.equal(torch.isinf(lse[live]), torch.isinf(l[live]))
        fine = torch.isfinite(l)
        assert float((lse.double() - l)[fine].abs().max() if fine.any() else 0.0) <= \
            z + 2.0 ** -20 * (1 + float(l[fine].abs().max() if fine.any() else 0))
        off = (out.double() - o).abs()[live]
        assert not bool(torch.isnan(off).any())
        worst = float((off / tol[live]).max()) if off.numel() else 0.0
        assert worst <= 1.0
        return out, lse

    def pool(self):
        conv = lambda t: (t.cpu().view(torch.int16).numpy().view(np.uint16)   # noqa: E731
                          if t.dtype == torch.bfloat16 else t.cpu().numpy())
        return O.KVPool(conv(self.kv.k_pages), conv(self.kv.v_pages), self.dtype,
                        None if self.kv.kv_scales is None else self.kv.kv_scales.cpu().numpy())

    def oracle(self):
        return O.chunk_attention(self.pool(), self.q.double().cpu().numpy(), self.offsets, self.lens,
                                 self.table, self.scale, self.window, self.sinks)


DTYPES = pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
MIXED = [(1, 1), (1, 17), (5, 5), (3, 40), (0, 9), (1, 300), (33, 64), (20, 100), (1, 16), (7, 3), (2, 0)]


@DTYPES
@pytest.mark.parametrize("window, sinks", [(0, 0), (1, 0), (10, 0), (32, 4), (33, 17), (50, 100), (64, 1)])
def test_mixed_batch(dtype, window, sinks):
    c = Chunks(dtype, MIXED, window=window, sinks=sinks)
    c.check()


@DTYPES
def test_the_reference_is_the_oracle(dtype):
    c = Chunks(dtype, MIXED, window=20, sinks=3)
    o, l, *_ = c.want()
    oo, ll = c.oracle()
    live = slice(0, int(c.offsets[-1]))
    assert np.allclose(o.cpu().numpy()[live], oo[live], atol=1e-9)
    assert np.array_equal(np.isinf(l.cpu().numpy()[live]), np.isinf(ll[live]))
    assert np.allclose(l.cpu().numpy()[live], ll[live], atol=1e-9)


@DTYPES
@pytest.mark.parametrize("Hq, Hkv, D", [(4, 4, 64), (6, 2, 64), (8, 1, 128), (3, 3, 128), (5, 1, 256),
                                        (32, 8, 128), (4, 2, 256), (40, 1, 64), (7, 7, 128)])
@pytest.mark.parametrize("window, sinks", [(0, 0), (40, 5)])
def test_head_layouts(dtype, Hq, Hkv, D, window, sinks):
    Chunks(dtype, [(1, 50), (9, 80), (70, 70), (1, 400), (130, 200)], Hq=Hq, Hkv=Hkv, D=D, window=window,
           sinks=sinks, seed=Hq + D).check()


@DTYPES
@pytest.mark.parametrize("n", [2, 8, 9, 31, 32, 33, 63, 64, 65, 127, 129, 257, 400])
def test_chunk_lengths(dtype, n):
    Chunks(dtype, [(n, n), (n, n + 1), (n, n + 77)], seed=n).check()


@DTYPES
@pytest.mark.parametrize("window, sinks", [(0, 0), (700, 0), (1000, 40), (5000, 4)])
def test_long_contexts(dtype, window, sinks):
    # decode rows split many ways, and chunks whose blocks are split
    Chunks(dtype, [(1, 20000), (300, 6000), (1, 31), (4, 9001), (1, 3000)], window=window, sinks=sinks,
           seed=window).check()


@DTYPES
@pytest.mark.parametrize("D, Hq, Hkv", [(128, 8, 2), (64, 8, 2), (256, 4, 1)])
def test_prompts(dtype, D, Hq, Hkv):
    Chunks(dtype, [(1500, 1500), (700, 900)], Hq=Hq, Hkv=Hkv, D=D, seed=7).check()
    Chunks(dtype, [(1500, 1500)], Hq=Hq, Hkv=Hkv, D=D, window=300, sinks=6, seed=8).check()


@DTYPES
@pytest.mark.parametrize("B", [64, 65, 130, 1025, 2100])
def test_many_sequences(dtype, B):
    rng = np.random.default_rng(B)
    seqs = [(int(n), int(n + c)) for n, c in zip(rng.choice([0, 1, 1, 1, 2, 6], B), rng.integers(0, 90, B))]
    Chunks(dtype, seqs, Hq=4, Hkv=1, D=64, seed=B).check()


@DTYPES
@pytest.mark.parametrize("kind", ["decode", "short", "all"])
@pytest.mark.parametrize("D, Hkv", [(64, 2), (128, 2), (128, 8), (256, 2)])
@pytest.mark.parametrize("window, sinks", [(0, 0), (100, 20)])
def test_servers(dtype, kind, D, Hkv, window, sinks):
    # more than 64 sequences: blocks of all rows, of teams and of wavefronts by themselves in one
    # launch, split and whole
    Chunks(dtype, server_batch(kind), Hq=4 * Hkv, Hkv=Hkv, D=D, window=window, sinks=sinks, seed=D + Hkv).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("seqs", [[(1, 17), (5, 40), (1, 900), (9, 1000), (30, 31)], [(1, 20000)],
                                  server_batch("short")])
@pytest.mark.parametrize("D, window", [(64, 0), (128, 0), (256, 0), (128, 70)])
def test_weights_of_few_rows_keep_16_bits(dtype, seqs, D, window):
    # up to 128 rows a sequence: each weight is off by 2^-8 of 2^-8 (two parts of bf16), and
    # the output is rounded once
    c = Chunks(dtype, seqs, Hkv=2, D=D, window=window, seed=21)
    out, _ = c.run()
    o, _, mean, far, most = c.want()
    z = (D + 4) * 2.0 ** -24 * abs(c.scale) * far
    near = mean * (2 * z + most * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -16) + most * 8 * 2.0 ** -118
    tol = near + 2.0 ** -8 * (o.abs() + near)
    live = int(c.offsets[-1])
    assert bool(((out.double() - o).abs() <= tol)[:live].all())


@DTYPES
def test_random_batches(dtype):
    rng = np.random.default_rng(12)
    for i in range(12):
        seqs = []
        for _ in range(int(rng.integers(1, 9))):
            n = int(rng.choice([0, 1, 1, 2, 5, 17, 60, 250]))
            seqs.append((n, max(0, n + int(rng.choice([-3, 0, 1, 15, 100, 1000])))))
        w = int(rng.choice([0, 0, 1, 16, 100, 1000]))
        Chunks(dtype, seqs, Hq=8, Hkv=int(rng.choice([1, 2, 8])), D=int(rng.choice([64, 128])), window=w,
               sinks=int(rng.choice([0, 0, 1, 33, 200])) if w else 0, seed=100 + i, pad=i % 3).check()


@DTYPES
def test_windows_as_verify(dtype):
    # the same windows through kap_verify (outputs in float32 there)
    c = Chunks(dtype, [(5, 200), (5, 77), (5, 5), (5, 1000)], pad=0)
    out, lse = c.check()
    o, l = K.verify(c.kv, c.q.view(4, 5, 8, 128), dev_i32(c.lens), dev_i32(c.table), c.most, c.scale)
    assert torch.allclose(lse.view(4, 5, 8), l, atol=1e-4)
    assert torch.allclose(out.view(4, 5, 8, 128).float(), o, atol=1e-4 if dtype == "f32" else 0.03)


@DTYPES
@pytest.mark.parametrize("scale, spread", [(-0.1, 1.0), (0.0, 1.0), (1.0, 3.0), (30.0, 1.0)])
def test_scales(dtype, scale, spread):
    Chunks(dtype, [(1, 900), (40, 300), (200, 333)], scale=scale, spread=spread, seed=4).check()


@DTYPES
def test_pages_outside_the_pool(dtype):
    for window, sinks in ((0, 0), (100, 20)):
        c = Chunks(dtype, [(1, 500), (60, 300), (150, 400), (3, 30)], window=window, sinks=sinks, seed=5)
        c.table[0, [3, 20]] = [-1, 2 ** 31 - 1]
        c.table[1, 5] = c.kv.num_pages
        c.table[2, [0, 7, 8, 9]] = [-2 ** 31, -1, -1, -7]
        c.table[3, :] = -1                                         # nothing is left of it
        out, lse = c.check()
        r = int(c.offsets[3])
        assert bool((lse[r:r + 3] == -math.inf).all()) and not bool(out[r:r + 3].any())


def poison(c, pages, t, value, which="v"):
    """Sets tokens of physical pages to a value (fp8: NaN's code)."""
    code = 0x7f if c.dtype == "fp8" else value
    for p in pages:
        if which == "v":
            c.kv.v_pages[p, :, :, t] = code
        else:
            c.kv.k_pages[p, :, :, t] = code


@DTYPES
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window, sinks", [(0, 0), (64, 8)])
def test_what_no_row_sees_may_hold_anything(dtype, value, window, sinks):
    # slots past a sequence's end, pages before its window, pages of no sequence
    c = Chunks(dtype, [(1, 37), (9, 200), (100, 250), (1, 1000), (300, 700)], window=window, sinks=sinks,
               seed=6)
    want = c.check()
    for b, (n, L) in enumerate(zip(c.new, c.lens)):
        for which in "kv":
            if L % 16:
                poison(c, [c.table[b, L // 16]], slice(L % 16, 16), value, which)
            if window:
                first = max(0, L - n - window + 1)                 # the lowest position in a window
                for j in range(-(-sinks // 16), first // 16):
                    poison(c, [c.table[b, j]], slice(0, 16), value, which)
    held = set(int(p) for b, L in enumerate(c.lens) for p in c.table[b, :-(-L // 16)])
    for p in set(range(c.kv.num_pages)) - held:
        poison(c, [p], slice(0, 16), value, "k")
        poison(c, [p], slice(0, 16), value, "v")
        if dtype == "fp8":
            c.kv.kv_scales[p] = value
    got = c.run()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_what_some_rows_see_reaches_those_alone(dtype, value):
    for seqs, b, pos, (window, sinks) in (([(40, 300)], 0, 280, (0, 0)), ([(9, 64), (1, 70)], 1, 3, (0, 0)),
                                          ([(200, 220)], 0, 100, (30, 4)), ([(200, 220)], 0, 2, (30, 4)),
                                          ([(300, 900)], 0, 450, (200, 0)), ([(1, 3000)], 0, 1500, (0, 0))):
        c = Chunks(dtype, seqs, window=window, sinks=sinks, seed=9)
        page = int(c.table[b, pos // 16])
        c.kv.v_pages[page, 1, 3, pos % 16] = value                 # one dim of one KV head
        out, lse = c.run()
        o, l = c.oracle()
        got = out.double().cpu().numpy()
        live = int(c.offsets[-1])
        for r in range(live):
            for h in range(8):
                w, g = o[r, h], got[r, h]
                assert np.array_equal(np.isnan(w), np.isnan(g)), (r, h)
                assert np.array_equal(w[np.isinf(w)], g[np.isinf(w)]), (r, h)
                f = np.isfinite(w)
                assert np.abs(w[f] - g[f]).max() < 0.05
        assert np.abs(lse.cpu().numpy()[:live] - l[:live]).max() < 1e-3


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan])
def test_infinite_and_nan_scales_of_seen_pages(scale):
    # values of ones under the scale: every row that sees the page gets it
    c = Chunks("fp8", [(1, 60), (5, 300), (200, 260), (4, 90)], seed=22)
    for b in range(3):
        c.kv.v_pages[int(c.table[b, 1])] = 0x38
        c.kv.kv_scales[int(c.table[b, 1]), 1] = scale
    want = Chunks("fp8", [(1, 60), (5, 300), (200, 260), (4, 90)], seed=22).run()
    out, lse = c.run()
    assert torch.equal(lse, want[1]) and torch.equal(out[206:], want[0][206:])
    assert bool((torch.isnan(out[:206]) if math.isnan(scale) else out[:206] == scale).all())


@DTYPES
def test_nan_in_a_query_and_in_a_seen_key(dtype):
    c = Chunks(dtype, [(5, 100), (40, 90), (1, 50)], seed=10)
    c.q[2, 3] = math.nan
    c.kv.k_pages[int(c.table[1, 4]), 0, 2, 5, 1] = 0x7f if dtype == "fp8" else math.nan   # position 69
    out, lse = c.run()
    bad = torch.zeros(c.T, 8, dtype=torch.bool, device="cuda")
    bad[2, 3] = True
    bad[5 + 69 - 50:45, :4] = True
    live = int(c.offsets[-1])
    assert torch.equal(torch.isnan(lse)[:live], bad[:live])
    assert torch.equal(torch.isnan(out).all(-1)[:live], bad[:live])
    assert torch.equal(torch.isnan(out).any(-1)[:live], bad[:live])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_climbing_logits(dtype):
    # every key above the ones before it, far apart: the reference moves all the time
    c = Chunks(dtype, [(1, 600), (80, 400)], Hq=2, Hkv=1, seed=11, scale=0.05)
    for b, L in enumerate(c.lens):
        for j in range(-(-L // 16)):
            k = torch.zeros(16, 128)
            k[:, 0] = torch.arange(16 * j, 16 * j + 16)
            c.kv.k_pages[int(c.table[b, j]), 0] = k.view(16, 16, 8).transpose(0, 1).to(c.q.dtype)
    c.q[:] = 0
    c.q[:, 0, 0], c.q[:, 1, 0] = 40.0, -40.0
    c.check()


@DTYPES
def test_the_workspace_holds_zero_counters_and_scratch(dtype):
    # one workspace for calls of several sizes, one after the other; the counters come back
    # zero, what is behind them does not matter
    calls = [Chunks(dtype, [(1, 8000), (260, 3000), (2, 500)], seed=13),
             Chunks(dtype, [(1, 900 + 40 * i) for i in range(70)], seed=14),
             Chunks(dtype, [(1, 20000)], Hq=2, Hkv=1, seed=15)]
    want = [c.run() for c in calls]
    need = max(K.chunk_attention_workspace_bytes(c.kv, len(c.lens), c.T, c.most) for c in calls)
    counters = 128 * torch.cuda.get_device_properties(0).multi_processor_count
    for seed in range(3):
        ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device="cuda",
                           generator=torch.Generator(device="cuda").manual_seed(seed))
        ws[:counters] = 0
        for c, w in zip(calls, want):
            for x, y in zip(c.run(workspace=ws), w):
                assert torch.equal(x, y)
            assert not bool(ws[:counters].any())


def test_without_lse():
    c = Chunks("bf16", [(1, 3000), (100, 200)], seed=14)
    want = c.run()[0]
    out = torch.full_like(c.q, FILL)
    ws = torch.zeros(K.chunk_attention_workspace_bytes(c.kv, 2, c.T, c.most), dtype=torch.uint8, device="cuda")
    off, lens, table = dev_i32(c.offsets), dev_i32(c.lens), dev_i32(c.table)
    import ctypes
    assert K.load_library().kap_chunk_attention(
        ctypes.byref(c.kv.struct), 2, c.T, c.q.data_ptr(), off.data_ptr(), lens.data_ptr(),
        table.data_ptr(), table.shape[1], c.most, 0, 0, c.scale, out.data_ptr(), None, ws.data_ptr(),
        ws.numel(), torch.cuda.current_stream().cuda_stream) == K.KAP_OK
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("window", [2 ** 31, 2 ** 32 + 5, -2 ** 32 + 5])
def test_windows_beyond_32_bits_are_none(window):
    c = Chunks("bf16", [(3, 90), (70, 400)])
    plain = c.run()
    c.window = window
    for got, want in zip(c.run(), plain):
        assert torch.equal(got, want)


def test_more_rows_than_tokens_under_the_longest_window():
    # tall blocks whose first rows are before position 0, a window just below the longest
    # length there is
    c = Chunks("bf16", [(700, 500)], Hq=32, Hkv=32, seed=20)
    plain = c.check()
    c.most = 2 ** 31 - 65
    table = np.full((1, -(-c.most // 16)), -5, np.int32)
    table[:, :c.table.shape[1]] = c.table
    c.table, c.window = table, c.most - 1
    for got, want in zip(c.run(), plain):
        assert torch.equal(got, want)


def test_nothing_to_do():
    for seqs in ([(0, 5), (0, 0)], [(1, 0)], [(3, 1)]):
        Chunks("bf16", seqs, seed=15).check()
    c = Chunks("bf16", [(0, 9)], pad=0)
    c.run()


@DTYPES
def test_captured_with_other_lengths(dtype):
    # lengths, tables and offsets change between replays; the sums of the plan with them
    c = Chunks(dtype, [(1, 700), (50, 120), (1, 90), (200, 460)], seed=16, wide=30)
    d = dict(off=dev_i32(c.offsets), lens=dev_i32(c.lens), table=dev_i32(c.table))
    out, lse = torch.full_like(c.q, FILL), torch.full(c.q.shape[:2], FILL, device="cuda")
    most = c.most + 64
    ws = torch.zeros(K.chunk_attention_workspace_bytes(c.kv, 4, c.T, most), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    call = K.bind_chunk_attention(c.kv, c.q, d["off"], d["lens"], d["table"], most, c.scale, out, lse, ws,
                                  stream=stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for new, lens in (([1, 50, 1, 200], [700, 120, 90, 460]), ([250, 0, 1, 1], [300, 5, 91, 1]),
                      ([1, 1, 1, 1], [16, 17, 15, 400]), ([0, 0, 252, 0], [0, 0, 96, 0])):
        c.new, c.lens = np.array(new), np.array(lens)
        c.offsets = np.concatenate([[0], np.cumsum(new)])
        d["off"].copy_(dev_i32(c.offsets)), d["lens"].copy_(dev_i32(c.lens))
        out.fill_(FILL), lse.fill_(FILL)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = c.run()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        c.check()


def test_two_calls_at_once():
    pairs = [(Chunks("bf16", [(1, 5000), (150, 800)], seed=s), torch.cuda.Stream()) for s in (17, 18)]
    want = [c.run() for c, _ in pairs]
    args = [(dev_i32(c.offsets), dev_i32(c.lens), dev_i32(c.table)) for c, _ in pairs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [K.chunk_attention(c.kv, c.q, *x, c.most, c.scale, stream=s)
               for (c, s), x in zip(pairs, args)]
        torch.cuda.synchronize()
        for (c, _), (o, l), w in zip(pairs, got, want):
            n = int(c.offsets[-1])
            assert torch.equal(o[:n], w[0][:n]) and torch.equal(l[:n], w[1][:n])


def test_pages_beyond_32_bit_offsets():
    small = Chunks("fp8", [(1, 900), (300, 500)], seed=19)
    n = small.kv.num_pages
    pages = (5 << 30) // (2 * 128 * 16) + n
    k, v = (torch.empty((pages, *t.shape[1:]), dtype=torch.uint8, device="cuda")
            for t in (small.kv.k_pages, small.kv.v_pages))
    sc = torch.ones((pages, 2), device="cuda")
    k[-n:], v[-n:], sc[-n:] = small.kv.k_pages, small.kv.v_pages, small.kv.kv_scales
    want = small.run()
    small.kv = K.KVCache(k, v, 8, torch.bfloat16, sc)
    small.table = small.table + (pages - n)
    for x, y in zip(small.run(), want):
        assert torch.equal(x, y)
