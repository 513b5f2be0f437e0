"""The calls of a continuous-batching step together, as a server makes them: block
tables and slots from the requests' lengths (kap_step_tables), keys, values and queries
turned and appended (kap_rope_append_kv), attention of prompts' chunks and single tokens
in one batch (kap_chunk_attention), penalties, biases and a grammar on the last row's
logits (kap_adjust_logits), and the draw (kap_sample), for several steps, eagerly and as
one captured graph. Every stage is compared with the oracle on the inputs that it had."""
import numpy as np
import pytest
import torch

from oracle import kap_oracle as O
from paper_2607_24260_amd import kap as K

from kap_testlib import LSE_TOL, assert_close, dev_i32
from test_gpu_rope_append import bits, check as check_append, make_pool
from test_gpu_sample import check as check_sample

pytestmark = pytest.mark.gpu

Hq, Hkv, D, VOCAB, B, T, CAP = 8, 2, 128, 997, 6, 400, 1200
# new tokens of the six sequences, step by step, and what they keep (None: all): prompts in
# chunks, single tokens, drafts taken back, a sequence that ends and another in its place
STEPS = [([300, 1, 40, 0, 7, 16], None), ([1, 80, 3, 5, 1, 1], None), ([3, 1, 1, 200, 0, 1], [None, 79, None, 2, None, 17]),
         ([1, 1, 1, 1, 33, 1], [301, None, 0, None, 0, None]), ([1, 1, 150, 4, 1, 1], None)]


class Server:
    def __init__(self, dtype, window, sinks, seed):
        self.dtype, self.window, self.sinks = dtype, window, sinks
        self.rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        pages, stride = 90, 40
        self.kv = make_pool(dtype, pages, Hq, Hkv, D, seed + 1)
        if dtype == "fp8":                       # (random codes: no NaN among them)
            for t in (self.kv.k_pages, self.kv.v_pages):
                t.masked_fill_((t & 127) == 127, 0x30)
        dt = self.kv.q_dtype
        i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(dtype=torch.float32, device="cuda")
        # what the host knows: lengths, tokens so far
        self.lens_n, self.history_n = np.zeros(B, np.int64), [[] for _ in range(B)]
        self.step = 0
        # what the device keeps
        self.lens, self.table = torch.zeros(B, **i32), torch.full((B, stride), -1, **i32)
        self.ring, self.free = dev_i32(self.rng.permutation(pages)), dev_i32([pages - 7, pages])
        self.history, self.told = torch.zeros((B, CAP), **i32), torch.zeros(B, **i32)
        self.start = torch.arange(B, device="cuda", dtype=torch.int64) * CAP
        self.most = 16 * stride
        # what a step is given
        self.add, self.keep = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.tokens = torch.zeros(T, dtype=torch.int64, device="cuda")
        self.last = torch.zeros(B, dtype=torch.int64, device="cuda")
        self.uniform = torch.zeros(B, **f32)
        self.embed = torch.randn((VOCAB, (Hq + 2 * Hkv) * D), generator=g, device="cuda").to(dt)
        self.order = torch.randperm(Hq * D, generator=g, device="cuda")[:VOCAB]
        self.inv = torch.as_tensor(1e4 ** (-np.arange(0, 64, 2) / 64), dtype=torch.float32).cuda()
        f = lambda v: torch.as_tensor(np.asarray(v, np.float32)).cuda()   # noqa: E731
        self.par = dict(prompt_len=dev_i32([300, 81, 40, 5, 7, 16]), repetition=f([1, 1.1, 1.3, 1, 1.2, 1]),
                        frequency=f([0, 0.5, 0, 0.2, 0, 1]), presence=f([0, 0.3, 0, 0, 0.1, 0]))
        words = self.rng.integers(0, 2 ** 32, (2, -(-VOCAB // 32)), dtype=np.uint64).astype(np.uint32)
        self.masks_n, self.mask_row_n = words, np.array([-1, 0, -1, 1, 0, -1])
        self.bias_n = [(3, 500.0), (900, -2.0), (3, 1.5), (17, 4.0)]
        self.par.update(bias_offsets=dev_i32([0, 0, 3, 3, 4, 4, 4]),
                        bias_token=dev_i32([t for t, _ in self.bias_n]), bias_value=f([v for _, v in self.bias_n]),
                        masks=torch.as_tensor(words.view(np.int32)).cuda(), mask_row=dev_i32(self.mask_row_n))
        self.temperature, self.top_k = torch.full((B,), 0.8, **f32), dev_i32([0, 5, 0, 40, 1, 0])
        self.top_p = torch.full((B,), 0.95, **f32)
        # what it leaves
        self.q_offsets, self.status = torch.zeros(B + 1, **i32), torch.zeros(B, **i32)
        self.slots, self.positions = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.zeros(T, **i32)
        self.x = torch.zeros((T, (Hq + 2 * Hkv) * D), dtype=dt, device="cuda")
        self.q = torch.zeros((T, Hq, D), dtype=dt, device="cuda")
        self.out, self.lse = torch.zeros((T, Hq, D), dtype=dt, device="cuda"), torch.zeros((T, Hq), **f32)
        self.raw, self.logits = torch.zeros((B, VOCAB), **f32), torch.zeros((B, VOCAB), **f32)
        self.token, self.prob = torch.zeros(B, **i32), torch.zeros(B, **f32)
        self.bad = torch.zeros(1, **i32)
        self.ws = torch.zeros(K.chunk_attention_workspace_bytes(self.kv, B, T, self.most, window=window,
                                                                sinks=sinks), dtype=torch.uint8, device="cuda")
        self.ws_sample = torch.zeros(max(256, K.sample_workspace_bytes(B, VOCAB)), dtype=torch.uint8,
                                     device="cuda")

    def feed(self):
        """The next step's lengths, tokens and histories."""
        add, keep = STEPS[self.step]
        self.step += 1
        add = np.array(add)
        keep = np.array([L if keep is None or keep[b] is None else keep[b] for b, L in enumerate(self.lens_n)])
        tokens, last = [], []
        for b in range(B):
            mine = self.rng.integers(0, 60, add[b]) * 13 % VOCAB
            self.history_n[b] = self.history_n[b][:keep[b]] + mine.tolist()
            tokens += mine.tolist()
            last.append(max(len(tokens) - 1, 0))
            self.history[b, :len(self.history_n[b])] = dev_i32(self.history_n[b])
        self.lens_n, self.keep_n, self.add_n = keep + add, keep, add
        self.keep.copy_(dev_i32(keep)), self.add.copy_(dev_i32(add)), self.told.copy_(dev_i32(self.lens_n))
        self.tokens.zero_()
        self.tokens[:len(tokens)] = torch.as_tensor(tokens).cuda()
        self.last.copy_(torch.as_tensor(last))
        self.uniform.copy_(torch.as_tensor(self.rng.random(B), dtype=torch.float32))

    def run(self, stream=None):
        K.step_tables(self.lens, self.add, self.table, self.ring, self.free, keep=self.keep,
                      free_out=self.free, new_lens=self.lens, q_offsets=self.q_offsets,
                      slot_mapping=self.slots, positions=self.positions, status=self.status, stream=stream)
        torch.index_select(self.embed, 0, self.tokens, out=self.x)
        q, k, v = self.parts()
        K.rope_append_kv(self.kv, k, v, self.slots, self.positions, self.inv, q_new=q, q_out=self.q,
                         bad_slots=self.bad, stream=stream)
        K.chunk_attention(self.kv, self.q, self.q_offsets, self.lens, self.table, self.most, D ** -0.5,
                          out=self.out, lse=self.lse, workspace=self.ws, window=self.window,
                          sinks=self.sinks, stream=stream)
        rows = torch.index_select(self.out.view(T, Hq * D), 0, self.last).float()
        torch.index_select(rows, 1, self.order, out=self.raw)
        self.raw.mul_(12.0)
        self.logits.copy_(self.raw)
        K.adjust_logits(self.logits, self.logits, history=self.history.view(-1), history_start=self.start,
                        history_len=self.told, stream=stream, **self.par)
        K.sample(self.logits, self.uniform, temperature=self.temperature, top_k=self.top_k, top_p=self.top_p,
                 token=self.token, prob=self.prob, workspace=self.ws_sample, stream=stream)

    def parts(self):
        return tuple(t.unflatten(1, (-1, D)) for t in self.x.split([Hq * D, Hkv * D, Hkv * D], 1))

    def before(self):
        host = lambda t: t.cpu().numpy().copy()                    # noqa: E731
        return dict(lens=host(self.lens), table=host(self.table), ring=host(self.ring), free=host(self.free),
                    pool=(bits(self.kv.k_pages), bits(self.kv.v_pages)), out=self.out.clone(), lse=self.lse.clone())

    def check(self, was):
        want = O.step_tables(was["lens"], self.add_n, was["table"], was["ring"], was["free"], T, keep=self.keep_n)
        for name, t in (("block_table", self.table), ("free_pages", self.ring), ("free_out", self.free),
                        ("new_lens", self.lens), ("q_offsets", self.q_offsets), ("slot_mapping", self.slots),
                        ("positions", self.positions), ("status", self.status)):
            assert np.array_equal(t.cpu().numpy().astype(np.int64), want[name]), name
        assert not want["status"].any() and np.array_equal(want["new_lens"], self.lens_n)
        q, k, v = self.parts()
        check_append(self.kv, self.dtype, q, k, v, self.slots.cpu().numpy(), self.positions, self.inv, None, False,
                     before=was["pool"], q_got=self.q, bad=self.bad)
        n = int(want["q_offsets"][-1])
        pool = O.KVPool(bits(self.kv.k_pages).view(np.uint16) if self.dtype == "bf16" else bits(self.kv.k_pages),
                        bits(self.kv.v_pages).view(np.uint16) if self.dtype == "bf16" else bits(self.kv.v_pages),
                        self.dtype, None if self.kv.kv_scales is None else self.kv.kv_scales.cpu().numpy())
        qd = self.q.double().cpu().numpy()
        args = (want["q_offsets"], self.lens_n, want["block_table"], D ** -0.5, self.window, self.sinks)
        o, l = O.chunk_attention(pool, qd, *args)
        # |V| in place of V: what roundings of the weights can move an output by
        size = O.chunk_attention(O.KVPool(pool.k_pages, pool.v_pages & 0x7f if self.dtype == "fp8" else
                                          (pool.v_pages & 0x7fff if self.dtype == "bf16" else np.abs(pool.v_pages)),
                                          self.dtype, pool.scales), qd, *args)[0]
        off = np.abs(self.out.double().cpu().numpy() - o)[:n]
        # half a step of bf16 for the weights and one for the output; 2e-3 is what the tests of
        # attention allow the sums and exponentials in 32 bits
        tol = 2e-3 if self.dtype == "f32" else 2.0 ** -8 * (size + np.abs(o))[:n] + 2e-3
        assert (off <= tol).all()
        assert_close("LSE", self.lse.cpu().numpy()[:n], l[:n], LSE_TOL, None)
        assert torch.equal(self.out[n:], was["out"][n:]) and torch.equal(self.lse[n:], was["lse"][n:])
        raw, got = self.raw.cpu().numpy(), self.logits.double().cpu().numpy()
        prompt = self.par["prompt_len"].cpu().numpy()
        for b in range(B):
            at = self.history_n[b]
            p = [float(self.par[k][b]) for k in ("repetition", "frequency", "presence")]
            biases = [self.bias_n[i] for i in range(*self.par["bias_offsets"][b:b + 2].tolist())]
            m = self.mask_row_n[b]
            allowed = None if m < 0 else np.unpackbits(self.masks_n[m].view(np.uint8), bitorder="little")[:VOCAB]
            w = O.adjust_logits(raw[b], at[:prompt[b]], at[prompt[b]:], *p, biases, allowed)
            assert np.array_equal(np.isinf(w), np.isinf(got[b]))
            f = np.isfinite(w)
            # five roundings in 32 bits of what is at most |x| r + f n + p + |bias|, and one more
            near = 6 * 2.0 ** -24 * (np.abs(raw[b]) * p[0] + p[1] * len(at) + p[2] + 500.0)
            assert (np.abs(got[b][f] - w[f]) <= near[f]).all()
        token, prob = check_sample(self.logits, self.uniform.cpu().numpy(), self.temperature.cpu().numpy(),
                                   self.top_k.cpu().numpy(), self.top_p.cpu().numpy())
        assert np.array_equal(token, self.token.cpu().numpy())
        assert np.array_equal(prob, self.prob.cpu().numpy())

    def state(self):
        return [self.kv.k_pages, self.kv.v_pages] + [getattr(self, name) for name in (
            "lens", "table", "ring", "free", "q_offsets", "slots", "positions", "status", "q", "out", "lse",
            "logits", "token", "prob")]


WINDOWS = pytest.mark.parametrize("window, sinks", [(0, 0), (48, 4)])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@WINDOWS
def test_steps(dtype, window, sinks):
    s = Server(dtype, window, sinks, 3)
    for _ in STEPS:
        s.feed()
        was = s.before()
        s.run()
        torch.cuda.synchronize()
        s.check(was)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "fp8"])
@WINDOWS
def test_a_captured_step_is_the_eager_one(dtype, window, sinks):
    eager, graphed = Server(dtype, window, sinks, 7), Server(dtype, window, sinks, 7)
    stream = torch.cuda.Stream()
    pools = graphed.kv.k_pages.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        graphed.run(stream)
    assert torch.equal(graphed.kv.k_pages, pools)         # capturing runs nothing
    for _ in STEPS:
        eager.feed(), graphed.feed()
        eager.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)


def test_two_servers_at_once_on_two_streams():
    # each with its own pool and workspaces, against the same one after the other
    pairs = [(Server("bf16", 0, 0, seed), Server("bf16", 0, 0, seed), torch.cuda.Stream()) for seed in (5, 6)]
    for _ in STEPS:
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
