"""GPU parity of kap_rope_append_kv with the oracle: Q, K and V of new tokens
turned by positions of one to four axes and written into the paged cache.

Tolerances. Let E = 2^-21 (|x| + |y|) for an output of the pair (x, y): the
remainder of the angle after whole quarter turns is rounded to 2^-26 quarters
(2.4e-8), sine and cosine are good to 2 ulp (2^-23 * 2), and two products and
a sum round by 2^-24 each: (2^-25 + 2^-22 + 3 * 2^-24) (|x| + |y|) < E. To that
comes the rounding to the stored type, at most half a step: bf16 2^-8 of the
value; E4M3FN 2^-4 of it, or 2^-10 below its smallest normal, after a division
(2^-24) by the page's scale.
"""
import numpy as np
import pytest
import torch

from oracle import kap_oracle as O
from paper_2607_24260_amd import kap as K

pytestmark = pytest.mark.gpu

QDT = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
F8 = torch.float8_e4m3fn


def make_pool(dtype, pages, Hq, Hkv, D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    shapes = ((pages, Hkv, D // 8, 16, 8), (pages, Hkv, D, 16))
    if dtype == "fp8":
        k, v = (torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8) for s in shapes)
        sc = torch.rand((pages, 2), generator=g, device="cuda") * 0.02 + 0.004
        return K.KVCache(k, v, Hq, torch.bfloat16, sc)
    k, v = (torch.randn(s, generator=g, device="cuda").to(QDT[dtype]) for s in shapes)
    return K.KVCache(k, v, Hq, QDT[dtype])


def numbers(t):
    return (t.view(F8) if t.dtype == torch.uint8 else t).double().cpu().numpy()


def half_step(dtype, want):
    if dtype == "f32":
        return 2.0 ** -24 * np.abs(want)
    if dtype == "bf16":
        return 2.0 ** -8 * np.abs(want)
    return np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10)


def spread(x, n, pairs):
    """2^-21 (|x| + |y|) of each dim's pair; nothing for dims that are not turned."""
    a, e = np.abs(x), np.zeros_like(x)
    for j in range(n):
        d0, d1 = (2 * j, 2 * j + 1) if pairs else (j, j + n)
        e[..., d0] = e[..., d1] = 2.0 ** -21 * (a[..., d0] + a[..., d1])
    return e


def check(kv, dtype, q, k, v, slots, pos, inv, axis, pairs, *, before, q_got, bad=None):
    pool = O.KVPool(before[0], before[1], dtype, None if kv.kv_scales is None
                    else kv.kv_scales.cpu().numpy())
    kd, vd = numbers(k), numbers(v)
    qd = None if q is None else numbers(q)
    ax = None if axis is None else axis.cpu().numpy()
    inv_n = inv.cpu().numpy()
    want_q, want_k, want_v, want_bad = O.rope_append_kv(pool, qd, kd, vd, slots, pos.cpu().numpy(),
                                                        inv_n, ax, pairs)
    n = len(inv_n)
    if q is not None:
        t = "f32" if dtype == "f32" else "bf16"
        got = numbers(q_got)
        assert np.all(np.abs(got - want_q) <= half_step(t, want_q) + spread(qd, n, pairs))
    if bad is not None:
        assert int(bad.item()) == want_bad
    # the same bound, placed like the values
    flat = O.KVPool(np.zeros_like(before[0], dtype=np.float64), np.zeros_like(before[1], dtype=np.float64),
                    "f32", None)
    scale = np.ones((pool.k_pages.shape[0], 2)) if pool.scales is None else pool.scales.astype(np.float64)
    spr, _ = O.append_kv(flat, spread(kd, n, pairs), np.zeros_like(vd), slots)
    for got, want, old, e, i in ((kv.k_pages, want_k, before[0], spr.k_pages, 0),
                                 (kv.v_pages, want_v, before[1], spr.v_pages, 1)):
        s = scale[:, i].reshape(-1, *[1] * (want.ndim - 1))
        got_n, live = numbers(got), ~np.isnan(want)
        tol = half_step(dtype, want) + e / s + 2.0 ** -23 * np.abs(want)
        if dtype != "fp8" and i == 1:
            tol = np.zeros_like(want)                        # V is copied
        assert np.all(np.abs(got_n - want)[live] <= tol[live])
        raw = got.view(torch.uint8) if got.dtype == torch.uint8 else got
        raw = raw.view(torch.int16) if raw.dtype == torch.bfloat16 else raw
        assert np.array_equal(raw.cpu().numpy()[~live], old[~live])   # the rest as it was


def bits(t):
    return (t.view(torch.int16) if t.dtype == torch.bfloat16 else t).cpu().numpy().copy()


def case(dtype, T, Hq, Hkv, D, rot, axes, pairs, seed, *, fused=True, runs=True, start=0, bad=True,
         with_q=True, shift=0):
    rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
    pages = (T + start) // 16 + 4
    kv = make_pool(dtype, pages, Hq, Hkv, D, seed + 1)
    w = (Hq + 2 * Hkv) * D
    buf = torch.randn(T * w + shift, generator=g, device="cuda").to(QDT[dtype])[shift:].view(T, w)
    q, k, v = (x.unflatten(1, (-1, D)) for x in buf.split([Hq * D, Hkv * D, Hkv * D], 1))
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    if runs:                                    # consecutive tokens, pages in any order
        order = rng.permutation(pages)
        at = start + np.arange(T)
        slots = (order[at // 16] * 16 + at % 16).astype(np.int64)
    else:
        slots = rng.choice(pages * 16, T, replace=False).astype(np.int64)
    if T > 4:
        slots[rng.integers(0, T, 2)] = -1
        if bad:
            slots[rng.integers(0, T)] = pages * 16 + int(rng.integers(0, 2**40))
    pos = rng.integers(0, 262144, (axes, T))
    pos[0, 0] = -3
    pos = torch.as_tensor(pos, dtype=torch.int32).cuda()
    inv = torch.as_tensor(1e6 ** (-np.arange(0, rot, 2) / rot), dtype=torch.float32).cuda()
    axis = None if axes == 1 else torch.as_tensor(rng.integers(-1, axes + 1, rot // 2),
                                                  dtype=torch.int32).cuda()
    before = bits(kv.k_pages), bits(kv.v_pages)
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    style = K.KAP_ROPE_PAIRS if pairs else K.KAP_ROPE_HALVES
    keep = buf.clone()
    got = K.rope_append_kv(kv, k, v, torch.as_tensor(slots).cuda(), pos, inv,
                           q_new=q if with_q else None, freq_axis=axis, style=style, bad_slots=count)
    torch.cuda.synchronize()
    assert torch.equal(buf, keep)               # the inputs are not touched
    check(kv, dtype, q if with_q else None, k, v, slots, pos, inv, axis, pairs, before=before,
          q_got=got, bad=count)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T, runs, start", [(1, True, 5), (3, True, 15), (16, True, 0), (17, False, 0),
                                            (40, True, 9), (150, True, 1), (130, False, 0)])
def test_tokens(dtype, pairs, T, runs, start):
    case(dtype, T, 8, 2, 128, 128, 1, pairs, 11 + T, runs=runs, start=start)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("Hq, Hkv, D, rot", [(3, 3, 64, 64), (12, 4, 64, 16), (32, 8, 128, 96),
                                             (5, 1, 256, 256), (16, 16, 256, 48), (6, 2, 128, 64)])
def test_heads_and_partial_rotation(dtype, Hq, Hkv, D, rot):
    case(dtype, 37, Hq, Hkv, D, rot, 3, False, 100 + rot, start=3)
    case(dtype, 37, Hq, Hkv, D, rot, 2, True, 200 + rot, fused=False, runs=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_rows_that_are_not_16_byte_aligned(dtype):
    case(dtype, 50, 4, 2, 64, 32, 4, False, 7, shift=1, start=2)
    case(dtype, 50, 4, 2, 128, 128, 1, True, 8, shift=3, with_q=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_long_chunk(dtype):
    case(dtype, 2100, 8, 2, 128, 128, 3, False, 21, start=7)


def test_in_place_queries():
    kv = make_pool("bf16", 4, 8, 2, 128, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((33, 8, 128), generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((33, 2, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in "kv")
    slots = torch.arange(33, device="cuda")
    pos = torch.arange(33, dtype=torch.int32, device="cuda")
    inv = torch.rand(64, generator=g, device="cuda")
    want = K.rope_append_kv(kv, k, v, slots, pos, inv, q_new=q)
    got = K.rope_append_kv(kv, k, v, slots, pos, inv, q_new=q, q_out=q)
    assert got is q and torch.equal(got, want)


def test_without_rotation_it_is_the_plain_append():
    # positions of zero: the stored bits are the inputs', as kap_append_kv's
    a, b = make_pool("bf16", 9, 8, 2, 128, 3), make_pool("bf16", 9, 8, 2, 128, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((100, 2, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in "kv")
    slots = torch.arange(20, 120, device="cuda")
    pos = torch.zeros(100, dtype=torch.int32, device="cuda")
    inv = torch.ones(64, device="cuda")
    K.rope_append_kv(a, k, v, slots, pos, inv)
    K.append_kv(b, k, v, slots)
    assert torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)


def test_values_that_are_not_finite_or_out_of_range_fp8():
    kv = make_pool("fp8", 2, 2, 1, 64, 5)
    kv.kv_scales.copy_(torch.tensor([[0.5, 0.25], [0.0, 0.0]]))
    k = torch.zeros((20, 1, 64), dtype=torch.bfloat16, device="cuda")
    k[:, 0, 40], k[:, 0, 41], k[:, 0, 42], k[:, 0, 43] = 1e30, -float("inf"), float("nan"), 300.0
    slots = torch.arange(20, device="cuda")
    pos = torch.zeros(20, dtype=torch.int32, device="cuda")
    inv = torch.ones(8, device="cuda")
    K.rope_append_kv(kv, k, k, slots, pos, inv)
    got_k = kv.k_pages.view(F8).float().permute(0, 3, 1, 2, 4).reshape(32, 64)[:20].cpu()
    got_v = kv.v_pages.view(F8).float().permute(0, 3, 1, 2).reshape(32, 64)[:20].cpu()
    for got in (got_k, got_v):
        assert torch.all(got[:, 40] == 448) and torch.all(got[:, 41] == -448)
        assert torch.all(torch.isnan(got[:, 42])) and torch.all(got[:, 43] == 448)
        assert torch.all(got[:16, :40] == 0)
        assert torch.all(torch.isnan(got[16:, :40]))         # 0 / 0: a page without a scale


def test_replayed_graph_and_other_stream():
    kv = make_pool("bf16", 40, 8, 2, 128, 6)
    g = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randn((64, 8, 128), generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn((64, 2, 128), generator=g, device="cuda").to(torch.bfloat16) for _ in "kv")
    slots = torch.arange(64, device="cuda") * 9
    pos = torch.arange(64, dtype=torch.int32, device="cuda")
    inv = torch.rand(64, generator=g, device="cuda")
    q_out = torch.zeros_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call = K.bind_rope_append_kv(kv, k, v, slots, pos, inv, q_new=q, q_out=q_out, stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
    for i in range(3):
        pos.add_(100 * i)
        kv.k_pages.zero_(), kv.v_pages.zero_(), q_out.zero_()
        want_kv = K.KVCache(kv.k_pages.clone(), kv.v_pages.clone(), 8, torch.bfloat16)
        want = K.rope_append_kv(want_kv, k, v, slots, pos, inv, q_new=q)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, want)
        assert torch.equal(kv.k_pages, want_kv.k_pages) and torch.equal(kv.v_pages, want_kv.v_pages)


def test_binding_refuses():
    kv = make_pool("bf16", 4, 8, 2, 128, 1)
    k = torch.zeros((6, 2, 128), dtype=torch.bfloat16, device="cuda")
    slots = torch.arange(6, device="cuda")
    pos = torch.zeros(6, dtype=torch.int32, device="cuda")
    inv = torch.ones(64, device="cuda")
    q = torch.zeros((6, 8, 128), dtype=torch.bfloat16, device="cuda")
    good = dict(kv=kv, k_new=k, v_new=k, slot_mapping=slots, positions=pos, inv_freq=inv)
    for over in (dict(k_new=k.float()), dict(v_new=k[:5]), dict(slot_mapping=slots.int()),
                 dict(positions=pos[:5]), dict(positions=pos.long()), dict(inv_freq=inv.double()),
                 dict(inv_freq=inv[:3]), dict(freq_axis=pos), dict(q_new=q.cpu()),
                 dict(q_new=q.transpose(1, 2).contiguous().transpose(1, 2)), dict(q_out=q),
                 dict(q_new=q, q_out=q[:5]), dict(k_new=k[:1].expand(6, 2, 128)), dict(style=5),
                 dict(positions=pos.expand(5, 6).contiguous())):
        with pytest.raises((ValueError, TypeError, K.KapError)):
            K.rope_append_kv(**{**good, **over})
    with pytest.raises(ValueError):
        K.bind_rope_append_kv(**good, q_new=q)
    assert K.rope_append_kv(kv, k[:0], k[:0], slots[:0], pos[:0], inv) is None


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("pairs", [False, True])
def test_an_angle_of_zero_leaves_infinities_alone(dtype, pairs):
    # positions of 0 on one axis, frequencies of an axis that is not there
    # (infinite ones among them): such pairs stay as they are, bit for bit
    T, D, n = 40, 128, 48
    kv = make_pool(dtype, 4, 4, 2, D, 30)
    g = torch.Generator(device="cuda").manual_seed(31)
    q, k, v = (torch.randn((T, h, D), generator=g, device="cuda").to(QDT[dtype]) for h in (4, 2, 2))
    for x in (q, k):
        at = torch.randint(0, x.numel(), (4 * T,), generator=g, device="cuda")
        x.view(-1)[at] = torch.tensor([float("inf"), -float("inf"), float("nan"), -0.0],
                                      device="cuda").to(x.dtype).repeat(T)
    axis = torch.arange(n, dtype=torch.int32, device="cuda") % 4 - 1       # -1, 0, 1, 2: two are there
    inv = torch.rand(n, generator=g, device="cuda")
    inv[axis == -1] = float("inf")
    pos = torch.stack([torch.arange(T, device="cuda") * 0, torch.arange(T, device="cuda") + 5]).int()
    slots = torch.arange(T, device="cuda") + 3
    got = K.rope_append_kv(kv, k, v, slots, pos, inv, q_new=q, freq_axis=axis,
                           style=K.KAP_ROPE_PAIRS if pairs else K.KAP_ROPE_HALVES)
    torch.cuda.synchronize()
    still = torch.ones(D, dtype=torch.bool)
    for j in range(n):
        if int(axis[j]) == 1:
            still[[2 * j, 2 * j + 1] if pairs else [j, j + n]] = False
    assert 0 < int(still[:2 * n].sum()) < 2 * n
    raw = lambda x: torch.where(torch.isnan(x), torch.nan, x).contiguous().view(
        torch.int32 if x.dtype == torch.float32 else torch.int16)
    assert torch.equal(raw(got[..., still]), raw(q[..., still]))
    at_slots = lambda p: p.permute(0, 3, 1, 2, 4).reshape(64, 2, D)[3:3 + T]
    if dtype == "fp8":
        scale = kv.kv_scales[:, 0].repeat_interleave(16)[3:3 + T, None, None]
        want = (k.float() / scale).clamp(-448, 448)[..., still]
        assert np.all(np.isnan(numbers(at_slots(kv.k_pages)[..., still])) == want.isnan().cpu().numpy())
        diff = np.abs(numbers(at_slots(kv.k_pages)[..., still]) - want.double().cpu().numpy())
        assert np.nanmax(diff / half_step("fp8", np.nan_to_num(want.double().cpu().numpy()))) <= 1 + 2.0 ** -20
    else:
        assert torch.equal(raw(at_slots(kv.k_pages)[..., still]), raw(k[..., still]))
