"""kap_step_tables against the oracle, entry for entry."""
import numpy as np
import pytest
import torch

from oracle import kap_oracle as O
from paper_2607_24260_amd import kap as K

from kap_testlib import dev_i32

pytestmark = pytest.mark.gpu

NAMES = ("block_table", "free_pages", "free_out", "new_lens", "q_offsets", "slot_mapping",
         "positions", "status")


def same(got, want):
    for name in NAMES:
        g = got[name].cpu().numpy().astype(np.int64)
        assert np.array_equal(g, want[name]), (name, g, want[name])


def call(lens, add, table, ring, state, T, keep=None, pinned=None, in_place=False, stream=None):
    opt = lambda x: None if x is None else dev_i32(x)              # noqa: E731
    table, ring, lens, state = dev_i32(table), dev_i32(ring), dev_i32(lens), dev_i32(state)
    more = dict(new_lens=lens, free_out=state) if in_place else {}
    got = K.step_tables(lens, dev_i32(add), table, ring, state, keep=opt(keep),
                        pinned_blocks=opt(pinned), num_tokens=T, stream=stream, **more)
    torch.cuda.synchronize()
    return dict(got, block_table=table, free_pages=ring)


def both(*args, **kw):
    want = O.step_tables(*args, **{k: v for k, v in kw.items() if k != "in_place"})
    same(call(*args, **kw), want)
    return want


def server(rng, B, ctx, spare=20, extra=0):
    lens = rng.integers(0, ctx + 1, B)
    have = -(-lens // 16)
    stride = int(have.max(initial=0)) + 8 + extra
    pages = int(have.sum()) + spare
    ids = rng.permutation(pages)
    table = np.full((B, stride), -1)
    at = 0
    for b in range(B):
        table[b, :have[b]] = ids[at:at + have[b]]
        at += have[b]
    head = int(rng.integers(0, pages))
    ring = np.full(pages, -1)
    ring[(head + np.arange(pages - at)) % pages] = ids[at:]
    return lens, table, ring, (head, pages - at)


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 1023, 1024, 1025, 2500])
def test_decode_steps(B):
    rng = np.random.default_rng(B)
    lens, table, ring, state = server(rng, B, 500, spare=B + 3)
    both(lens, np.ones(B, int), table, ring, state, B + 5)
    both(lens, np.ones(B, int), table, ring, state, B, in_place=True)


@pytest.mark.parametrize("B", [3, 70, 1030])
@pytest.mark.parametrize("seed", range(4))
def test_windows_prompts_and_ends(B, seed):
    rng = np.random.default_rng(10 * B + seed)
    lens, table, ring, state = server(rng, B, 300, spare=10 * B, extra=130)
    keep = np.where(rng.random(B) < 0.2, 0, lens - rng.integers(0, 9, B)).clip(0)
    add = np.where(rng.random(B) < 0.1, rng.integers(0, 2000, B), rng.integers(0, 6, B))
    pinned = rng.integers(-2, 5, B)
    T = int(add.sum())
    for n in (T, T + 100, max(T // 2, 1)):
        both(lens, add, table, ring, state, n, keep=keep, pinned=pinned, in_place=seed % 2 == 0)


def test_refusals_by_sequence():
    lens, add = [5, 5, 5, -1, 5, 31, 16, 3, 16], [1, -1, 1, 1, 28, 3, 1, 9, 1]
    keep = [5, 5, 6, 0, 5, 31, 16, 3, 16]
    table = np.arange(18).reshape(9, 2)
    for T in (0, 1, 9, 10, 11, 12, 400):
        for count in (0, 1, 2):
            both(lens, add, table, [90, 91], (1, count), T, keep=keep)
    low = -2 ** 31
    both([low, 40, 2 ** 31 - 1, 4], [3, low, 2 ** 31 - 1, 2 ** 31 - 1], np.zeros((4, 3)), [7, 8],
         (0, 2), 64, keep=[low, 40, 3, 4])


@pytest.mark.parametrize("state", [(-1, 3), (8, 3), (2, 9), (2, -4), (7, 8), (0, 0), (2 ** 31 - 1, 2 ** 31 - 1),
                                   (-2 ** 31, -2 ** 31)])
def test_odd_states_of_the_ring(state):
    table = np.arange(12).reshape(3, 4) + 100
    both([33, 5, 64], [1, 20, 0], table, np.arange(8), state, 30, keep=[20, 5, 0])
    both([0, 0, 0], [0, 0, 0], table, np.arange(8), state, 0)


def test_no_pages_no_tokens():
    both([0, 0], [0, 3], np.zeros((2, 2)), np.zeros(0, int), (0, 0), 4)
    both([0, 3], [0, 0], np.zeros((2, 0)), [4], (0, 1), 0)
    # the ring is full: what comes back is lost, as documented
    both([40, 0], [0, 0], [[1, 2, 3], [0, 0, 0]], [6, 7], (1, 2), 3, keep=[0, 0])


def test_a_step_of_no_sequence():
    got = call([], [], np.zeros((0, 4)), [5, 6, 7], (1, 2), 0)
    assert got["free_out"].tolist() == [1, 2] and got["q_offsets"].tolist() == [0]
    assert got["free_pages"].tolist() == [5, 6, 7]


@pytest.mark.parametrize("bound", [False, True])
@pytest.mark.parametrize("state", [(1, 2), (0, 3), (-1, 9), (3, -4), (2 ** 31 - 1, -2 ** 31)])
def test_a_step_of_no_sequence_in_arrays_that_are_there(bound, state):
    i32 = lambda *x: dev_i32(np.array(x, int))                     # noqa: E731
    out = dict(free_out=i32(77, 77), new_lens=i32(), q_offsets=i32(77), positions=i32(), status=i32(),
               slot_mapping=torch.zeros(0, dtype=torch.int64, device="cuda"))
    want = O.step_tables([], [], np.zeros((0, 4)), [5, 6, 7], state, 0)
    stream = torch.cuda.Stream()
    free = i32(*state)
    for other in (None, stream):
        for o in (out, dict(out, free_out=free)):                  # and in place
            o["free_out"].copy_(i32(77, 77)), o["q_offsets"].fill_(77), free.copy_(i32(*state))
            args = (i32(), i32(), torch.zeros((0, 4), dtype=torch.int32, device="cuda"), i32(5, 6, 7), free)
            torch.cuda.synchronize()
            if bound:
                K.bind_step_tables(*args, stream=other, **o)()
            else:
                K.step_tables(*args, stream=other, **o)
            torch.cuda.synchronize()
            assert o["free_out"].tolist() == list(want["free_out"]) and o["q_offsets"].tolist() == [0]


def test_long_prompts():
    # pages by the thousand for one sequence; slots of a second launch
    rng = np.random.default_rng(5)
    lens, table, ring, state = server(rng, 6, 40, spare=9000, extra=8000)
    both(lens, [1, 70000, 0, 4097, 1, 1], table, ring, state, 80000)
    both(lens, [0, 0, 0, 0, 0, 100000], table, ring, state, 100000)
    back = np.where(np.arange(6) == 1, 0, 3)
    want = O.step_tables(lens, [0, 120000, 0, 0, 0, 0], table, ring, state, 120000)
    both(want["new_lens"], back, want["block_table"], want["free_pages"], want["free_out"], 20,
         keep=np.where(np.arange(6) == 1, 0, want["new_lens"]))


def test_a_captured_step_follows_the_state():
    # lengths and the ring in place: replays go on where the last one ended
    rng = np.random.default_rng(8)
    B, T = 40, 200
    lens, table, ring, state = server(rng, B, 200, spare=400, extra=40)
    d = dict(lens=dev_i32(lens), add=dev_i32(np.zeros(B)), keep=dev_i32(lens), table=dev_i32(table),
             ring=dev_i32(ring), state=dev_i32(state))
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")   # noqa: E731
    out = dict(free_out=d["state"], new_lens=d["lens"], q_offsets=i32(B + 1),
               slot_mapping=torch.zeros(T, dtype=torch.int64, device="cuda"), positions=i32(T),
               status=i32(B))
    stream = torch.cuda.Stream()
    step = K.bind_step_tables(d["lens"], d["add"], d["table"], d["ring"], d["state"], keep=d["keep"],
                              stream=stream, **out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    want = dict(block_table=table, free_pages=ring, new_lens=lens, free_out=state)
    for i in range(5):
        keep = (want["new_lens"] - rng.integers(0, 4, B)).clip(0)
        add = rng.integers(0, 6, B)
        d["keep"].copy_(dev_i32(keep)), d["add"].copy_(dev_i32(add))
        want = O.step_tables(want["new_lens"], add, want["block_table"], want["free_pages"],
                             want["free_out"], T, keep=keep)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same(dict(out, block_table=d["table"], free_pages=d["ring"]), want)
