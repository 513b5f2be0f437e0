"""Refusals of the calls of a continuous-batching step -- kap_step_tables,
kap_chunk_attention, kap_adjust_logits -- before anything is enqueued (no GPU: fake pointers are never
dereferenced on those paths)."""
import ctypes
import os

import pytest

from paper_2607_24260_amd import kap as K

FAKE = 0x1000000
BAD, UNS = K.KAP_ERR_INVALID_ARGUMENT, K.KAP_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(K.LIB_PATH):
        pytest.fail("libkap.so is not built; run __graft_entry__.build() first")
    return K.load_library()


def tables(lib, **over):
    a = dict(B=4, lens=FAKE, keep=FAKE, add=FAKE, pinned=FAKE, table=FAKE, stride=64, ring=FAKE, size=100,
             state=FAKE, T=20, out=FAKE, new=FAKE, off=FAKE, slots=FAKE, pos=FAKE, status=FAKE)
    assert set(over) <= set(a)
    a.update(over)
    return lib.kap_step_tables(*a.values(), None)


@pytest.mark.parametrize("over, status", [
    (dict(B=-1), BAD), (dict(B=65536), UNS), (dict(stride=-1), BAD), (dict(stride=1 << 27), UNS),
    (dict(size=-1), BAD), (dict(T=-1), BAD), (dict(T=1 << 30), UNS), (dict(B=0), BAD),
    *[({k: None}, BAD) for k in ("lens", "add", "table", "ring", "state", "out", "new", "off", "slots", "pos",
                                 "status")],
    *[({k: FAKE + 2}, BAD) for k in ("lens", "keep", "add", "pinned", "table", "ring", "state", "out", "new",
                                     "off", "pos", "status")],
    (dict(slots=FAKE + 4), BAD),
])
def test_step_tables_refuses(lib, over, status):
    assert tables(lib, **over) == status
    assert lib.kap_last_error()


def test_step_tables_of_nothing(lib):
    assert tables(lib, B=0, T=0, lens=None, add=None, status=None) == K.KAP_OK
    assert lib.kap_last_error() == b""


def adjust(lib, **over):
    a = dict(rows=4, vocab=1000, x=FAKE, stride=1000, dt=K.KAP_DT_BF16, out=2 * FAKE, ostride=1000,
             history=FAKE, size=50, start=FAKE, len=FAKE, prompt=FAKE, rep=FAKE, freq=FAKE, pres=FAKE,
             boff=FAKE, btok=FAKE, bval=FAKE, biases=9, masks=FAKE, nmasks=3, mstride=32, mrow=FAKE)
    assert set(over) <= set(a)
    a.update(over)
    return lib.kap_adjust_logits(*a.values(), None)


@pytest.mark.parametrize("over, status", [
    (dict(rows=-1), BAD), (dict(rows=65536), UNS), (dict(vocab=0), BAD),
    (dict(vocab=1 << 30, stride=1 << 30, ostride=1 << 30), BAD), (dict(dt=K.KAP_DT_FP8_E4M3FN), UNS),
    (dict(stride=999), BAD), (dict(ostride=999), BAD), (dict(stride=2 ** 61), UNS), (dict(ostride=2 ** 61), UNS),
    (dict(size=-1), BAD), (dict(biases=-1), BAD), (dict(nmasks=-1), BAD), (dict(mstride=31), BAD),
    (dict(mstride=2 ** 60), UNS), (dict(x=None), BAD), (dict(out=None), BAD), (dict(start=None), BAD),
    (dict(len=None), BAD), (dict(btok=None), BAD), (dict(bval=None), BAD), (dict(mrow=None), BAD),
    (dict(x=FAKE + 1), BAD), (dict(out=FAKE + 1), BAD), (dict(x=FAKE + 2, dt=K.KAP_DT_F32), BAD),
    (dict(start=FAKE + 4), BAD),
    *[({k: FAKE + 2}, BAD) for k in ("history", "len", "prompt", "rep", "freq", "pres", "boff", "btok", "bval",
                                     "masks", "mrow")],
    # out over logits, but for logits themselves
    (dict(out=FAKE, ostride=1001), BAD), (dict(out=FAKE + 2), BAD), (dict(out=FAKE + 7998), BAD),
    (dict(out=FAKE - 7998), BAD),
])
def test_adjust_logits_refuses(lib, over, status):
    assert adjust(lib, **over) == status
    assert lib.kap_last_error()


def test_adjust_logits_of_no_rows(lib):
    assert adjust(lib, rows=0, x=None, out=None) == K.KAP_OK
    assert lib.kap_last_error() == b""


def kv_struct(kv_dtype=K.KAP_DT_BF16, q_dtype=K.KAP_DT_BF16, Hq=32, Hkv=8, D=128, page=16, scales=None,
              num_pages=100):
    return K.KVCacheStruct(Hq, Hkv, D, page, kv_dtype, q_dtype, FAKE, FAKE, scales, num_pages)


def chunk(lib, kv=None, **over):
    a = dict(B=4, T=20, q=FAKE, off=FAKE, lens=FAKE, table=FAKE, stride=64, most=1024, window=0, sinks=0,
             scale=1.0, out=2 * FAKE, lse=FAKE, ws=FAKE, have=None)
    assert set(over) <= set(a)
    a.update(over)
    kv = kv or kv_struct()
    have = a.pop("have")
    if have is None:
        have = lib.kap_chunk_attention_workspace_bytes(ctypes.byref(kv), a["B"], a["T"], a["most"],
                                                       a["window"], a["sinks"])
    return lib.kap_chunk_attention(ctypes.byref(kv), *a.values(), have, None)


@pytest.mark.parametrize("over, status", [
    (dict(B=-1), BAD), (dict(B=65536), UNS), (dict(B=0), BAD), (dict(T=-1), BAD), (dict(T=1 << 25), UNS),
    (dict(most=-1), BAD), (dict(stride=63), BAD), (dict(most=2 ** 31 - 64, stride=1 << 27), UNS),
    (dict(sinks=-1), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("-inf")), BAD),
    *[({k: None}, BAD) for k in ("q", "off", "lens", "table", "out")],
    (dict(q=FAKE + 8), BAD), (dict(out=FAKE + 8), BAD),
    *[({k: FAKE + 2}, BAD) for k in ("off", "lens", "table", "lse")],
    (dict(out=FAKE), BAD), (dict(out=FAKE + 16), BAD), (dict(out=FAKE - 20 * 32 * 128 * 2 + 16), BAD),
    (dict(ws=None), K.KAP_ERR_WORKSPACE_TOO_SMALL), (dict(have=1000), K.KAP_ERR_WORKSPACE_TOO_SMALL),
    (dict(ws=FAKE + 128), BAD),
])
def test_chunk_attention_refuses(lib, over, status):
    assert chunk(lib, **over) == status
    assert lib.kap_last_error()


def test_chunk_attention_pools_and_nothing(lib):
    assert chunk(lib, kv_struct(page=32)) == UNS
    assert chunk(lib, kv_struct(D=96)) == UNS
    assert chunk(lib, kv_struct(num_pages=0)) == BAD
    assert chunk(lib, kv_struct(kv_dtype=K.KAP_DT_FP8_E4M3FN)) == BAD
    assert chunk(lib, B=0, T=0, q=None, off=None, lens=None, table=None) == K.KAP_OK
    assert chunk(lib, T=0, q=None, out=None) == K.KAP_OK
    assert lib.kap_last_error() == b""
    size = lib.kap_chunk_attention_workspace_bytes
    kv = kv_struct()
    assert size(ctypes.byref(kv), 0, 5, 1024, 0, 0) == size(ctypes.byref(kv), 4, -1, 1024, 0, 0) == 0
    assert size(ctypes.byref(kv), 4, 5, 1024, 0, -1) == size(ctypes.byref(kv_struct(D=96)), 4, 5, 9, 0, 0) == 0
    assert 0 < size(ctypes.byref(kv), 4, 5, 1024, 100, 4) <= size(ctypes.byref(kv), 4, 5, 1024, 0, 0)
