"""kap_adjust_logits against the oracle.

An output goes through at most five operations in 32 bits (a quotient or product,
a product and two differences, a sum), each off by half a step of what it gives, which
is at most M = max(r, 1/r) |x| + f n + |p| + |bias|, and is rounded once: off by
at most 5 * 2^-24 M + half a step of the type at the result and what it is off by.
"""
import math

import numpy as np
import pytest
import torch

from oracle import kap_oracle as O
from paper_2607_24260_amd import kap as K

from kap_testlib import dev_i32

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


class Call:
    """Rows with histories in one array (start, length, prompt), lists of biases, masks."""

    def __init__(self, rows, vocab, dtype, seed, longest=200, told=True, biased=True, masked=True):
        rng = self.rng = np.random.default_rng(seed)
        self.rows, self.vocab, self.dtype = rows, vocab, dtype
        self.x = torch.as_tensor(rng.standard_normal((rows, vocab)) * 4).to(DT[dtype]).cuda()
        self.kw, self.host = {}, {}
        if told:
            n = rng.integers(0, longest + 1, rows)
            history = rng.integers(0, max(2, min(vocab, 40)), int(n.sum()) + 7) * 7919 % max(vocab, 1)
            start = np.concatenate([[0], np.cumsum(n)[:-1]])
            f = lambda v: np.asarray(v, np.float32)                # noqa: E731
            self.set(history=history, history_start=start, history_len=n,
                     prompt_len=rng.integers(-3, longest + 3, rows),
                     repetition=f(rng.choice([1.0, 0.8, 1.1, 1.5], rows)),
                     frequency=f(rng.choice([0.0, 0.3, -0.2], rows)),
                     presence=f(rng.choice([0.0, 0.7, -0.4], rows)))
        if biased:
            count = rng.choice([0, 1, 5, 60], rows)
            offs = np.concatenate([[0], np.cumsum(count)])
            self.set(bias_offsets=offs, bias_token=rng.integers(-2, vocab + 2, offs[-1] + 1),
                     bias_value=np.asarray(rng.uniform(-9, 5, offs[-1] + 1), np.float32))
        if masked:
            words = rng.integers(0, 2 ** 32, (4, -(-vocab // 32)), dtype=np.uint64).astype(np.uint32)
            words[0] = 0
            self.set(masks=words, mask_row=rng.integers(-2, 6, rows))

    def set(self, **kw):
        for k, v in kw.items():
            v = np.asarray(v)
            self.host[k] = v
            if v.dtype == np.uint32:
                self.kw[k] = torch.as_tensor(v.view(np.int32)).cuda()
            elif v.dtype == np.float32:
                self.kw[k] = torch.as_tensor(v).cuda()
            else:
                self.kw[k] = dev_i32(v) if k != "history_start" else torch.as_tensor(
                    v.astype(np.int64)).cuda()

    def want(self):
        h, xs = self.host, self.x.float().cpu().numpy()
        want, off = np.empty(xs.shape), np.empty(xs.shape)
        for r in range(self.rows):
            prompt, told, rep, freq, pres = [], [], 1.0, 0.0, 0.0
            if "history" in h:
                s, n = int(h["history_start"][r]), int(h["history_len"][r])
                cut = int(h["prompt_len"][r]) if "prompt_len" in h else 0
                for i in range(max(0, -s), min(n, len(h["history"]) - s)):
                    (prompt if i < cut else told).append(h["history"][s + i])
                rep, freq, pres = (float(h[k][r]) if k in h else d for k, d in
                                   (("repetition", 1.0), ("frequency", 0.0), ("presence", 0.0)))
            biases = []
            if "bias_offsets" in h:
                lo, hi = h["bias_offsets"][r:r + 2].clip(0, len(h["bias_token"]))
                biases = list(zip(h["bias_token"][lo:hi], h["bias_value"][lo:hi]))
            allowed = None
            if "masks" in h and 0 <= h["mask_row"][r] < len(h["masks"]):
                allowed = np.unpackbits(h["masks"][h["mask_row"][r]].view(np.uint8),
                                        bitorder="little")[:self.vocab]
            with np.errstate(invalid="ignore"):                    # (inf - inf)
                want[r] = O.adjust_logits(xs[r], prompt, told, rep, freq, pres, biases, allowed)
            off[r] = np.abs(xs[r]) * max(rep, 1 / rep) + abs(freq) * len(told) + abs(pres) + max(
                [abs(b) for _, b in biases], default=0)
        return want, off

    def check(self, out=None, **kw):
        want, size = self.want()
        before = self.x.clone()
        y = K.adjust_logits(self.x, out, **self.kw, **kw)
        torch.cuda.synchronize()
        raw = lambda t: t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
        if out is None:
            assert torch.equal(raw(self.x), raw(before))
        got = y.double().cpu().numpy()
        fine = np.isfinite(want)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        inf = np.isinf(want)
        assert np.array_equal(got[inf], want[inf])
        got, want, near = got[fine], want[fine], 5 * 2.0 ** -24 * size[fine]
        assert (np.abs(got - want) <= near + HALF[self.dtype] * (np.abs(want) + near)).all()
        return y


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab", [(1, 1), (3, 2), (7, 31), (5, 33), (9, 64), (6, 1000), (5, 8191),
                                         (4, 8193), (3, 32000), (3, 50021)])
def test_sizes(dtype, rows, vocab):
    Call(rows, vocab, dtype, vocab).check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", [(), ("told",), ("biased",), ("masked",), ("told", "masked")])
def test_parts(dtype, which):
    on = {k: k in which for k in ("told", "biased", "masked")}
    c = Call(5, 9001, dtype, 3, **on)
    y = c.check()
    if not which:
        assert torch.equal(y, c.x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_optional_arrays(dtype):
    for gone in (["prompt_len"], ["repetition"], ["frequency", "presence"], ["repetition", "presence"]):
        c = Call(4, 500, dtype, 4)
        for k in gone:
            del c.kw[k], c.host[k]
        c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_windows_share_a_history(dtype):
    c = Call(15, 700, dtype, 5)
    start = np.repeat([0, 50, 200], 5)
    c.set(history_start=start, history_len=30 + np.tile(np.arange(5), 3), prompt_len=np.repeat([10, 0, 40], 5))
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ranges_outside_the_lists(dtype):
    c = Call(9, 300, dtype, 6)
    n = len(c.host["history"])
    big = 2 ** 62
    c.set(history_start=np.array([-5, n - 3, n, big, -big, -(2 ** 63), 2 ** 63 - 1, 0, 3]),
          history_len=np.array([9, 10, 4, 5, 5, 5, 5, -7, 2 ** 31 - 1]),
          prompt_len=np.array([7, 1, 2, 3, 2 ** 31 - 1, 0, 0, 0, -2 ** 31]))
    c.set(bias_offsets=np.array([-9, 4, 2, 20, 10 ** 9, 5, 6, 6, 8, 2 ** 31 - 1]))
    c.set(history=np.where(np.arange(n) % 5 == 0, c.rng.choice([-1, 300, 2 ** 31 - 1, -2 ** 31], n),
                           c.host["history"]))
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_token_over_and_over(dtype):
    c = Call(4, 40, dtype, 7, longest=3)
    c.set(history=np.concatenate([np.full(70000, 17), np.full(300, 3)]), history_start=[0, 0, 69990, 0],
          history_len=[70000, 69999, 310, 70300], prompt_len=[0, 69998, 5, 69000],
          frequency=np.array([1e-3, 1.0, 0.5, -1e-4], np.float32))
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_nan_and_zeros(dtype):
    c = Call(6, 400, dtype, 8)
    pick = torch.randint(0, 9, c.x.shape, generator=torch.Generator().manual_seed(1)).cuda()
    for i, v in enumerate((math.inf, -math.inf, math.nan, 0.0, -0.0)):
        c.x[pick == i] = v
    c.check()


def test_parameters_that_are_not_used_may_be_anything():
    # a token that was not put out, of a row without its history: nothing of them comes in
    c = Call(3, 100, "f32", 9, biased=False, masked=False)
    c.set(history_len=[0, 0, 4], prompt_len=[0, 0, 4], frequency=np.array([math.inf, math.nan, math.nan], np.float32),
          presence=np.array([math.nan, math.inf, math.inf], np.float32),
          repetition=np.array([math.nan, 0.0, 1.0], np.float32))
    y = K.adjust_logits(c.x, **c.kw)
    assert torch.equal(y, c.x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [997, 1000, 8200])
def test_in_place_and_rows_apart(dtype, vocab):
    for pad_in, pad_out, shift_in, shift_out in ((0, 0, 0, 0), (3, 3, 1, 1), (5, 2, 1, 3), (0, 8, 0, 0), (1, 9, 2, 2)):
        c = Call(6, vocab, dtype, 11)
        big = torch.full((6 * (vocab + pad_in) + 9,), 77.0, dtype=DT[dtype], device="cuda")
        view = big[shift_in:shift_in + 6 * (vocab + pad_in)].view(6, -1)[:, :vocab]
        view.copy_(c.x)
        c.x = view
        out = torch.full((6 * (vocab + pad_out) + 9,), 55.0, dtype=DT[dtype], device="cuda")
        o = out[shift_out:shift_out + 6 * (vocab + pad_out)].view(6, -1)[:, :vocab]
        apart = c.check(o).clone()
        o.fill_(55.0)
        assert bool((out == 55.0).all()) and int((big == 77.0).sum()) >= 6 * pad_in + 9
        assert torch.equal(c.check(c.x), apart)                     # in place
        view.fill_(77.0)
        assert bool((big == 77.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_named_more_than_once_in_a_list(dtype):
    # the last entry counts, however far apart they are; lists longer than a workgroup
    c = Call(4, 5000, dtype, 14, biased=False)
    token = np.concatenate([np.arange(5000), [3, 3, 9], c.rng.integers(0, 5000, 3000), [4999] * 300, [7]])
    c.set(bias_token=token, bias_value=np.asarray(c.rng.uniform(-9, 5, len(token)), np.float32),
          bias_offsets=np.array([0, 5000, 5003, len(token) - 1, len(token)]))
    c.check()


def slice_of(rows, vocab, dtype):
    """Tokens of a workgroup: 16 KB of logits, halved while that leaves compute units idle."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    most = 8192 if dtype == "bf16" else 4096
    size = most
    while size > most // 8 and rows * -(-vocab // size) < 2 * cus:
        size //= 2
    return size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("part", [1, 2, 4, 8])
@pytest.mark.parametrize("slices, odd", [(8, 1), (1, -3)])
def test_slices_of_every_size(dtype, part, slices, odd):
    # as many rows as make the slice a whole, a half, .. of the largest
    most = 8192 if dtype == "bf16" else 4096
    size, vocab = most // part, slices * most + most // 2 + odd
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    rows = -(-2 * cus // -(-vocab // size)) if part < 8 else 3
    assert slice_of(rows, vocab, dtype) == size
    c = Call(rows, vocab, dtype, 20 + part, longest=900)
    n = len(c.host["history"])
    # tokens all over the vocabulary, some of them often; lists that name some twice
    c.set(history=np.where(c.rng.random(n) < 0.3, c.rng.integers(0, 9, n) * (vocab // 9), c.rng.integers(-2, vocab + 2, n)))
    lists = c.rng.choice([0, 3, 700], rows)
    offs = np.concatenate([[0], np.cumsum(lists)])
    pool = c.rng.integers(-2, vocab + 2, 3000)
    c.set(bias_offsets=offs, bias_token=c.rng.choice(pool, offs[-1]) if part % 4 else c.rng.permutation(offs[-1]) % vocab,
          bias_value=np.asarray(c.rng.uniform(-9, 5, offs[-1]), np.float32))
    plain = c.check()
    for pad, shift in ((0, 0), (5, 3)):
        big = torch.full((rows * (vocab + pad) + 9,), 77.0, dtype=DT[dtype], device="cuda")
        view = big[shift:shift + rows * (vocab + pad)].view(rows, -1)[:, :vocab]
        view.copy_(c.x)
        K.adjust_logits(view, view, **c.kw)                         # in place
        assert torch.equal(view, plain)
        view.fill_(77.0)
        assert bool((big == 77.0).all())
        out = torch.full((rows * (vocab + pad + 1) + 9,), 55.0, dtype=DT[dtype], device="cuda")
        o = out[shift:shift + rows * (vocab + pad + 1)].view(rows, -1)[:, :vocab]
        assert torch.equal(K.adjust_logits(c.x, o, **c.kw), plain)
        o.fill_(55.0)
        assert bool((out == 55.0).all())


def test_results_do_not_depend_on_the_run():
    c = Call(8, 30000, "bf16", 12, longest=5000)
    first = K.adjust_logits(c.x, **c.kw)
    for _ in range(5):
        assert torch.equal(K.adjust_logits(c.x, **c.kw), first)


def test_captured_with_a_growing_history():
    c = Call(4, 5000, "f32", 13)
    out = torch.zeros_like(c.x)
    stream = torch.cuda.Stream()
    call = K.bind_adjust_logits(c.x, out, stream=stream, **c.kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for i in range(4):
        c.kw["history_len"].add_(1)
        c.kw["masks"].bitwise_xor_(1 << i)
        eager = K.adjust_logits(c.x, **c.kw)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
