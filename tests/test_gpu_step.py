"""The calls of a serving step together: proposed tokens' keys and values turned
and appended (kap_rope_append_kv), attention over a batch whose sequences share
leading pages (kap_verify_shared), tokens drawn from the logits (kap_sample) and
the window accepted (kap_accept_top3), for several cycles, eagerly and as one
captured graph. Every stage is compared with the oracle on the inputs that it had."""
import numpy as np
import pytest
import torch

from oracle import kap_oracle as O
from paper_2607_24260_amd import kap as K

from kap_testlib import LSE_TOL, O_TOL, assert_close, dev_i32
from test_gpu_rope_append import bits, check as check_append, make_pool
from test_gpu_sample import check as check_sample

pytestmark = pytest.mark.gpu

Hq, Hkv, D, VOCAB = 8, 2, 128, 997
LEFT = ("q", "out", "lse", "token", "prob", "accepted", "carry")      # what a step leaves


class Server:
    """Five sequences, the first four a group that shares six pages, the third of
    them ending within a page; a model whose projections are rows of a table and
    whose logits are attention outputs in another order."""

    def __init__(self, dtype, window, seed):
        self.dtype, self.w, self.B, self.cycles = dtype, window, 5, 3
        rng, g = np.random.default_rng(seed), torch.Generator(device="cuda").manual_seed(seed)
        self.lens = np.array([96 + 3, 96 + 16, 96 + 45, 96 + 80, 33])
        most = 96 + 80 + self.cycles * window
        per = -(-most // 16)
        pages = 6 + self.B * per
        perm = rng.permutation(pages)
        self.table_n = perm[6:].reshape(self.B, per).copy()
        self.table_n[:4, :6] = perm[:6]
        self.kv = make_pool(dtype, pages, Hq, Hkv, D, seed + 1)
        if dtype == "fp8":                       # (random codes: no NaN among them)
            for t in (self.kv.k_pages, self.kv.v_pages):
                t.masked_fill_((t & 127) == 127, 0x30)
        self.most, self.table = most, dev_i32(self.table_n)
        self.offsets, self.blocks = dev_i32(np.array([0, 4])), dev_i32(np.array([6]))
        dt = self.kv.q_dtype
        T = self.T = self.B * window
        self.embed = torch.randn((VOCAB, (Hq + 2 * Hkv) * D), generator=g, device="cuda").to(dt)
        self.order = torch.randperm(Hq * D, generator=g, device="cuda")[:VOCAB]
        self.inv = torch.as_tensor(1e4 ** (-np.arange(0, 64, 2) / 64), dtype=torch.float32).cuda()
        self.axis = dev_i32(rng.integers(0, 2, 32))
        i32 = dict(dtype=torch.int32, device="cuda")
        f32 = dict(dtype=torch.float32, device="cuda")
        # what a cycle is given
        self.tokens = torch.randint(0, VOCAB, (T,), generator=g, device="cuda")
        self.slots = torch.zeros(T, dtype=torch.int64, device="cuda")
        self.positions, self.total = torch.zeros((2, T), **i32), torch.zeros(self.B, **i32)
        self.uniform, self.drafts = torch.rand(T, generator=g, device="cuda"), torch.zeros((self.B, window - 1), **i32)
        self.temperature = torch.full((T,), 0.8, **f32)
        self.top_k = dev_i32(rng.integers(0, 40, T))
        self.top_p = torch.full((T,), 0.95, **f32)
        # what it leaves
        self.x = torch.zeros((T, (Hq + 2 * Hkv) * D), dtype=dt, device="cuda")
        self.q = torch.zeros((T, Hq, D), dtype=dt, device="cuda")
        self.out, self.lse = torch.zeros((self.B, window, Hq, D), **f32), torch.zeros((self.B, window, Hq), **f32)
        self.logits = torch.zeros((T, VOCAB), **f32)
        self.token, self.prob = torch.zeros(T, **i32), torch.zeros(T, **f32)
        self.accepted, self.carry = torch.zeros(self.B, **i32), torch.zeros(self.B, **i32)
        self.bad = torch.zeros(1, **i32)
        space = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
        self.ws_attention = space(K.verify_shared_workspace_bytes(self.kv, self.B, window, most, 1))
        self.ws_sample = space(K.sample_workspace_bytes(T, VOCAB))
        self.ws_accept = torch.zeros(K.load_library().kap_accept_top3_workspace_bytes(self.B, window),
                                     dtype=torch.uint8, device="cuda")   # (zeroed once, kap.h)

    def parts(self):
        return tuple(t.unflatten(1, (-1, D)) for t in self.x.split([Hq * D, Hkv * D, Hkv * D], 1))

    def feed(self):
        """The next window of every sequence."""
        at = self.lens[:, None] + np.arange(self.w)[None, :]
        slots = np.take_along_axis(self.table_n, at // 16, 1) * 16 + at % 16
        self.slots.copy_(torch.as_tensor(slots.reshape(-1)))
        self.positions.copy_(torch.as_tensor(np.stack([at.reshape(-1), at.reshape(-1) // 7])))
        self.total.copy_(torch.as_tensor(self.lens + self.w))
        self.drafts.copy_(self.tokens.view(self.B, self.w)[:, 1:])

    def run(self, stream=None):
        torch.index_select(self.embed, 0, self.tokens, out=self.x)
        q, k, v = self.parts()
        K.rope_append_kv(self.kv, k, v, self.slots, self.positions, self.inv, q_new=q, q_out=self.q,
                         freq_axis=self.axis, bad_slots=self.bad, stream=stream)
        K.verify_shared(self.kv, self.q.view(self.B, self.w, Hq, D), self.total, self.table, self.most,
                        self.offsets, self.blocks, D ** -0.5, out=self.out, lse=self.lse,
                        workspace=self.ws_attention, stream=stream)
        torch.index_select(self.out.view(self.T, Hq * D), 1, self.order, out=self.logits)
        self.logits.mul_(12.0)
        K.sample(self.logits, self.uniform, temperature=self.temperature, top_k=self.top_k,
                 top_p=self.top_p, token=self.token, prob=self.prob, workspace=self.ws_sample,
                 stream=stream)
        K.accept_top3(self.logits.view(self.B, self.w, VOCAB), self.drafts, accepted=self.accepted,
                      carry=self.carry, workspace=self.ws_accept, stream=stream)

    def advance(self):
        """Accepted tokens stay; the next window is the carry token and draws."""
        torch.cuda.synchronize()
        self.lens = self.lens + np.minimum(self.accepted.cpu().numpy() + 1, self.w)
        nxt = self.token.view(self.B, self.w).clone()
        nxt[:, 0] = self.carry
        self.tokens.copy_(nxt.view(-1))
        self.uniform.copy_(torch.rand(self.T, generator=torch.Generator(device="cuda").manual_seed(
            int(self.lens.sum())), device="cuda"))

    def state(self):
        return [self.kv.k_pages, self.kv.v_pages] + [getattr(self, name) for name in LEFT]

    def check(self, before):
        q, k, v = self.parts()
        check_append(self.kv, self.dtype, q, k, v, self.slots.cpu().numpy(), self.positions, self.inv,
                     self.axis, False, before=before, q_got=self.q, bad=self.bad)
        conv = lambda t: (t.cpu().view(torch.int16).numpy().view(np.uint16)
                          if t.dtype == torch.bfloat16 else t.cpu().numpy())
        pool = O.KVPool(conv(self.kv.k_pages), conv(self.kv.v_pages), self.dtype,
                        None if self.kv.kv_scales is None else self.kv.kv_scales.cpu().numpy())
        o, l = O.verify(pool, self.q.view(self.B, self.w, Hq, D).double().cpu().numpy(),
                        self.total.cpu().numpy(), self.table_n, D ** -0.5)
        assert_close("O", self.out.cpu().numpy(), o, O_TOL, None)
        assert_close("LSE", self.lse.cpu().numpy(), l, LSE_TOL, None)
        # (draws of this size have no boundary within rounding but for one in 2^20)
        token, prob = check_sample(self.logits, self.uniform.cpu().numpy(),
                                   self.temperature.cpu().numpy(), self.top_k.cpu().numpy(),
                                   self.top_p.cpu().numpy())
        assert np.array_equal(token, self.token.cpu().numpy())
        assert np.array_equal(prob, self.prob.cpu().numpy())
        m, carry = O.accept_top_k(self.logits.view(self.B, self.w, VOCAB).cpu().numpy(),
                                  self.drafts.cpu().numpy())
        assert np.array_equal(self.accepted.cpu().numpy(), m)
        assert np.array_equal(self.carry.cpu().numpy(), carry)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("window", [1, 5])
def test_cycles(dtype, window):
    s = Server(dtype, window, 31 + window)
    for _ in range(s.cycles):
        s.feed()
        before = bits(s.kv.k_pages), bits(s.kv.v_pages)
        s.run()
        torch.cuda.synchronize()
        s.check(before)
        s.advance()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_a_captured_step_is_the_eager_one(dtype):
    eager, graphed = Server(dtype, 5, 77), Server(dtype, 5, 77)
    stream = torch.cuda.Stream()
    graphed.feed()
    pools = graphed.kv.k_pages.clone(), graphed.kv.v_pages.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        graphed.run(stream)
    assert torch.equal(graphed.kv.k_pages, pools[0])      # capturing runs nothing
    for _ in range(eager.cycles):
        eager.feed(), graphed.feed()
        eager.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)
        eager.advance(), graphed.advance()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
def test_two_steps_at_once_on_two_streams(dtype):
    # each with its own pool and workspaces, against the same one after the other
    pairs = [(Server(dtype, 5, seed), Server(dtype, 5, seed), torch.cuda.Stream()) for seed in (5, 6)]
    for _ in range(3):
        for alone, together, _ in pairs:
            alone.feed(), together.feed()
            alone.run()
            torch.cuda.synchronize()
        for _, together, stream in pairs:
            with torch.cuda.stream(stream):
                together.run(stream)
        torch.cuda.synchronize()
        for alone, together, _ in pairs:
            for a, b in zip(alone.state(), together.state()):
                assert torch.equal(a, b)
            alone.advance(), together.advance()


def test_pages_beyond_32_bit_offsets():
    # the same step in a pool of 9.8 GB, whose last pages it uses, and in a small one
    small = Server("fp8", 5, 41)
    n = small.kv.k_pages.shape[0]
    far = Server("fp8", 5, 41)
    pages = (5 << 30) // (Hkv * D * 16) + n
    shift = pages - n
    k, v = (torch.empty((pages, *t.shape[1:]), dtype=torch.uint8, device="cuda")
            for t in (small.kv.k_pages, small.kv.v_pages))
    scales = torch.ones((pages, 2), device="cuda")
    k[shift:], v[shift:], scales[shift:] = small.kv.k_pages, small.kv.v_pages, small.kv.kv_scales
    far.kv = K.KVCache(k, v, Hq, torch.bfloat16, scales)
    far.table = far.table + shift
    for _ in range(2):
        small.feed(), far.feed()
        far.slots += 16 * shift
        small.run(), far.run()
        torch.cuda.synchronize()
        assert torch.equal(k[shift:], small.kv.k_pages) and torch.equal(v[shift:], small.kv.v_pages)
        for a, b in ((getattr(small, x), getattr(far, x)) for x in LEFT):
            assert torch.equal(a, b)
        small.advance(), far.advance()
