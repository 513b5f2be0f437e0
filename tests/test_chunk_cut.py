"""How kap_chunk_attention's work is cut, on the host: the steps that rows walk against a
plain count, and what the cut of any batch keeps to -- as many workgroups as are launched,
counters and rows of partial results as the workspace has."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2607_24260_amd import build as B

from kap_testlib import server_batch

HERE = os.path.dirname(os.path.abspath(__file__))
I32, I64 = ctypes.c_int32, ctypes.c_int64
F32, BF16, FP8 = 0, 1, 2


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("cut") / "chunk_cut.so")
    r = subprocess.run([B.hipcc(), "--offload-host-only", "-x", "hip", "-O1", "-std=c++17", "-fPIC", "-shared",
                        f"-I{B.INCLUDE}", f"-I{B.CSRC}", os.path.join(HERE, "c", "chunk_cut.hip"), "-o", path],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return ctypes.CDLL(path)


def walked(lib, n, length, G, most, window, sinks, r0, r1):
    res = (I32 * 3)()
    lib.chunk_range(*map(I32, (n, length, G, most, window, sinks, r0, r1)), res)
    return tuple(res)


def seen_steps(n, length, G, window, sinks, r0, r1):
    """What rows [r0, r1) have to walk, in whole numbers of any size: the steps of 32 that
    hold sinks, and those from the lowest position in a window to the highest one."""
    p0, p1 = length - n + r0 // G, length - n + (r1 - 1) // G
    hi = max(0, p1 + 1)
    lo = max(0, p0 - window + 1) if window else 0
    start = min(lo, hi) // 32
    first = min(-(-min(sinks, hi) // 32), start) if window else 0
    return first, start, first + -(-hi // 32) - start


def test_ranges(lib):
    rng = np.random.default_rng(0)
    for _ in range(4000):
        G = int(rng.integers(1, 12))
        n = int(rng.integers(1, 400))
        length = int(rng.choice([n, n + 1, n + 500, max(0, n - 70), 0, 31, 32]))
        window = int(rng.choice([0, 1, 31, 32, 33, 100, 1000]))
        sinks = int(rng.choice([0, 1, 33, 200]))
        rows = n * G
        r0 = int(rng.integers(0, rows))
        r1 = min(rows, r0 + int(rng.choice([1, 32, 128, 256])))
        want = seen_steps(n, length, G, window, sinks, r0, r1)
        assert walked(lib, n, length, G, 2000, window, sinks, r0, r1) == want


KINDS = [(F32, 64), (F32, 128), (F32, 256), (BF16, 64), (BF16, 128), (BF16, 256), (FP8, 128), (FP8, 256)]


def batches(rng):
    """Sequences of (new tokens, length): decoding, prompts, both, many, uneven ones."""
    log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))   # noqa: E731
    kind = rng.integers(0, 6)
    ctx = log(1, 200000)
    B = log(1, 3000) if kind in (3, 4) else log(1, 100)
    seqs = []
    for b in range(B):
        if kind == 0 or (kind == 2 and b % 4) or (kind == 4 and b > 3):
            n = 1
        elif kind == 3:
            n = int(rng.choice([0, 1, 2, 30, 33, 130]))
        elif kind == 5:
            n = log(1, 20000) if b == 0 else int(rng.integers(0, 3))
        else:
            n = log(1, 4000)
        seqs.append((n, max(0, n + int(rng.integers(-2, ctx)))))
    return seqs


def check(lib, kv, D, Hq, Hkv, seqs, window, sinks, cus, pad=0, most=None):
    new = np.array([n for n, _ in seqs], np.int64)
    off = np.ascontiguousarray(np.concatenate([[0], np.cumsum(new)]), np.int32)
    lens = np.ascontiguousarray([L for _, L in seqs], np.int32)
    T, most = int(off[-1]) + pad, most or max(1, int(lens.max()))
    res = (I64 * 13)()
    i32 = ctypes.POINTER(I32)
    lib.chunk_cut(*map(I32, (kv, D, Hq, Hkv, len(seqs), T)), off.ctypes.data_as(i32), lens.ctypes.data_as(i32),
                  *map(I32, (most, window, sinks, cus)), res)
    (planned, tall, team, solo, whole, merged, rows, wrong, last, grid, counters, part_rows,
     part_lse) = res
    assert wrong == 0 and last < grid, (tall, team, solo, grid)
    assert merged <= counters and rows <= part_rows and rows <= part_lse, (merged, counters, rows, part_rows)
    G, wave_rows = Hq // Hkv, 32 * (4 if D == 256 or (kv == F32 and D == 128) else 8)
    blocks = lambda size: int(sum(-(-n * G // size) for n in new)) * Hkv       # noqa: E731
    assert blocks(wave_rows) <= whole <= blocks(32)
    if not planned:
        assert tall + team <= -(-max(whole, cus) // cus) * cus and solo == 0
    return planned, tall, team, solo, merged


@pytest.mark.parametrize("kv, D", KINDS)
def test_the_cut_of_any_batch_fits(lib, kv, D):
    rng = np.random.default_rng(D + kv)
    met = np.zeros(5, int)
    for i in range(150):
        seqs = batches(rng)
        Hkv = int(rng.choice([1, 2, 8]))
        window = int(rng.choice([0, 0, 1, 100, 4096]))
        r = check(lib, kv, D, Hkv * int(rng.choice([1, 4, 5])), Hkv, seqs, window, int(rng.choice([0, 4, 100])),
                  int(rng.choice([256, 256, 304, 8])), pad=int(rng.choice([0, 0, 50])),
                  most=int(rng.choice([0, 0, 300000])) or None)
        met += np.array(r) > 0
    # every kind was there: planned calls, tall parts, teams', solo ones, merges
    few = kv == F32 and D == 256
    assert met[0] and met[2] and met[3] and met[4] and (met[1] or few), met


@pytest.mark.parametrize("n, length, G, r0, r1", [
    (700, 500, 1, 0, 256),            # 200 rows that see nothing, 56 that see 1 to 56 keys
    (200, 120, 1, 0, 128), (2 ** 30 - 1, 5, 1, 0, 256), (2 ** 30 - 1, 5, 1, 2 ** 30 - 33, 2 ** 30 - 1)])
@pytest.mark.parametrize("window", [1, 100, 2 ** 30, 2 ** 31 - 300, 2 ** 31 - 66])
def test_ranges_of_long_windows_and_more_rows_than_tokens(lib, n, length, G, r0, r1, window):
    most = 2 ** 31 - 65               # the longest there is; windows below it are not "none"
    want = seen_steps(n, length, G, window, 0, r0, r1)
    assert walked(lib, n, length, G, most, window, 0, r0, r1) == want
    want = seen_steps(n, length, G, window, 40, r0, r1)
    assert walked(lib, n, length, G, most, window, 40, r0, r1) == want


@pytest.mark.parametrize("kv, D", KINDS)
@pytest.mark.parametrize("Hkv", [2, 8])
@pytest.mark.parametrize("window, sinks", [(0, 0), (100, 20)])
def test_the_kinds_of_the_batches_that_are_compared(lib, kv, D, Hkv, window, sinks):
    # what the batches of test_gpu_chunk_attention.test_servers are there for
    few = kv == F32 and D == 256                                   # (no tall blocks)
    got = {k: check(lib, kv, D, 4 * Hkv, Hkv, server_batch(k), window, sinks, 256) for k in ("decode", "short", "all")}
    assert all(planned for planned, *_ in got.values())
    _, tall, team, solo, merged = got["decode"]
    assert (tall > 0) != few and (team > 0 or window > 0)
    if not window and Hkv == 2 and (D == 64 or few):
        assert merged > 0
    _, tall, team, solo, merged = got["short"]
    assert tall == 0 and solo > 0 and (team > 0) == (D == 64 and not window and Hkv == 2 or
                                                     (kv, D, Hkv, window) in ((BF16, 128, 2, 0), (FP8, 128, 2, 0)))
    _, tall, team, solo, merged = got["all"]
    assert (tall > 0) != few and solo > 0 and (team > 0) != (window > 0)
