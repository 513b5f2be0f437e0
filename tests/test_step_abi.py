"""Refusals of the calls around a step -- kap_rope_append_kv, kap_verify_shared,
kap_sample -- before anything is enqueued (no GPU: fake pointers are never
dereferenced on those paths)."""
import ctypes
import os

import pytest

from paper_2607_24260_amd import kap as K

FAKE = 0x100000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(K.LIB_PATH):
        pytest.fail("libkap.so is not built; run __graft_entry__.build() first")
    return K.load_library()


def kv_struct(kv_dtype=K.KAP_DT_BF16, q_dtype=K.KAP_DT_BF16, Hq=32, Hkv=8, D=128, page=16,
              scales=None, num_pages=100):
    return K.KVCacheStruct(Hq, Hkv, D, page, kv_dtype, q_dtype, FAKE, FAKE, scales, num_pages)


def rope(lib, kv=None, **over):
    a = dict(T=5, q=FAKE, qs=4096, qo=8 * FAKE, k=2 * FAKE, ks=1024, v=3 * FAKE, vs=1024, slots=FAKE,
             pos=FAKE, axes=1, inv=FAKE, fa=None, rot=128, style=0, bad=None)
    assert set(over) <= set(a)
    a.update(over)
    kv = kv or kv_struct()
    return lib.kap_rope_append_kv(ctypes.byref(kv), a["T"], a["q"], a["qs"], a["qo"], a["k"],
                                  a["ks"], a["v"], a["vs"], a["slots"], a["pos"], a["axes"],
                                  a["inv"], a["fa"], a["rot"], a["style"], a["bad"], None)


BAD, UNS = K.KAP_ERR_INVALID_ARGUMENT, K.KAP_ERR_UNSUPPORTED


@pytest.mark.parametrize("over, status", [
    (dict(T=-1), BAD), (dict(axes=0), BAD), (dict(axes=5), BAD), (dict(rot=0), BAD),
    (dict(rot=24), BAD), (dict(rot=144), BAD), (dict(style=2), BAD), (dict(k=None), BAD),
    (dict(v=None), BAD), (dict(slots=None), BAD), (dict(pos=None), BAD), (dict(inv=None), BAD),
    (dict(q=None), BAD), (dict(qo=None), BAD), (dict(qs=4095), BAD), (dict(ks=1023), BAD),
    (dict(vs=1), BAD), (dict(qs=2**62), UNS), (dict(vs=2**60), UNS), (dict(T=2**30), UNS),
    (dict(k=2 * FAKE + 1), BAD), (dict(slots=FAKE + 4), BAD), (dict(pos=FAKE + 2), BAD),
    (dict(fa=FAKE + 1), BAD), (dict(qo=8 * FAKE + 8), BAD),
    # q_out over an input, except q itself where its rows are contiguous
    (dict(qo=FAKE, qs=4096 + 2048), BAD), (dict(qo=FAKE + 4096), BAD),
    (dict(qo=2 * FAKE + 16), BAD), (dict(qo=3 * FAKE - 16, T=1), BAD),
])
def test_rope_append_refuses(lib, over, status):
    assert rope(lib, **over) == status
    assert lib.kap_last_error()


def test_rope_append_refuses_pools(lib):
    assert rope(lib, kv_struct(page=32)) == UNS
    assert rope(lib, kv_struct(D=96), rot=96) == UNS
    assert rope(lib, kv_struct(kv_dtype=K.KAP_DT_F32)) == UNS
    assert rope(lib, kv_struct(kv_dtype=K.KAP_DT_FP8_E4M3FN)) == BAD
    assert b"kv_scales" in lib.kap_last_error()
    assert rope(lib, kv_struct(num_pages=0)) == BAD
    assert rope(lib, T=0, q=None, qo=None, k=None, v=None, slots=None, pos=None, inv=None) == K.KAP_OK
    assert lib.kap_last_error() == b""


def draw(lib, **over):
    a = dict(rows=4, vocab=1000, x=FAKE, stride=1000, dt=K.KAP_DT_BF16, t=FAKE, k=FAKE, p=FAKE, q=FAKE,
             u=FAKE, token=FAKE, prob=FAKE, ws="enough", have=None)
    assert set(over) <= set(a)
    a.update(over)
    need = lib.kap_sample_workspace_bytes(max(a["rows"], 0), max(a["vocab"], 0))
    ws = FAKE if a["ws"] == "enough" else a["ws"]
    have = need if a["have"] is None else a["have"]
    return lib.kap_sample(a["rows"], a["vocab"], a["x"], a["stride"], a["dt"], a["t"], a["k"], a["p"],
                          a["q"], a["u"], a["token"], a["prob"], ws, have, None)


@pytest.mark.parametrize("over, status", [
    (dict(rows=-1), BAD), (dict(vocab=0), BAD), (dict(vocab=1 << 30, stride=1 << 30), BAD),
    (dict(dt=K.KAP_DT_FP8_E4M3FN), UNS), (dict(stride=999), BAD), (dict(rows=65536), UNS),
    (dict(stride=2**61), UNS), (dict(x=None), BAD), (dict(u=None), BAD), (dict(token=None), BAD),
    (dict(x=FAKE + 1), BAD), (dict(x=FAKE + 2, dt=K.KAP_DT_F32), BAD), (dict(t=FAKE + 2), BAD),
    (dict(k=FAKE + 1), BAD), (dict(prob=FAKE + 2), BAD),
    (dict(ws=None), K.KAP_ERR_WORKSPACE_TOO_SMALL), (dict(have=99), K.KAP_ERR_WORKSPACE_TOO_SMALL),
    (dict(ws=FAKE + 64), BAD),
])
def test_sample_refuses(lib, over, status):
    assert draw(lib, **over) == status
    assert lib.kap_last_error()


def test_sample_of_no_rows(lib):
    assert draw(lib, rows=0, x=None, u=None, token=None) == K.KAP_OK
    assert lib.kap_sample_workspace_bytes(0, 1000) == lib.kap_sample_workspace_bytes(4, 0) == 0


def shared(lib, kv=None, **over):
    a = dict(B=4, w=5, q=FAKE, lens=FAKE, table=FAKE, stride=64, most=1024, groups=2, off=FAKE, blocks=FAKE,
             scale=1.0, out=FAKE, lse=FAKE, ws=FAKE, have=None)
    assert set(over) <= set(a)
    a.update(over)
    kv = kv or kv_struct()
    have = a["have"]
    if have is None:
        have = lib.kap_verify_shared_workspace_bytes(ctypes.byref(kv), a["B"], a["w"], a["most"],
                                                     a["groups"])
    return lib.kap_verify_shared(ctypes.byref(kv), a["B"], a["w"], a["q"], a["lens"], a["table"],
                                 a["stride"], a["most"], a["groups"], a["off"], a["blocks"],
                                 a["scale"], a["out"], a["lse"], a["ws"], have, None)


@pytest.mark.parametrize("over, status", [
    (dict(B=-1), BAD), (dict(B=65536), UNS), (dict(w=0), BAD), (dict(w=17), BAD), (dict(most=-1), BAD),
    (dict(stride=63), BAD), (dict(groups=-1), BAD), (dict(groups=5), BAD), (dict(q=None), BAD),
    (dict(lens=None), BAD), (dict(table=None), BAD), (dict(off=None), BAD), (dict(blocks=None), BAD),
    (dict(out=None), BAD), (dict(lse=None), BAD), (dict(scale=float("nan")), BAD),
    (dict(scale=float("inf")), BAD), (dict(q=FAKE + 8), BAD), (dict(out=FAKE + 4), BAD),
    (dict(ws=None), K.KAP_ERR_WORKSPACE_TOO_SMALL), (dict(have=1000), K.KAP_ERR_WORKSPACE_TOO_SMALL),
    (dict(ws=FAKE + 128), BAD),
])
def test_verify_shared_refuses(lib, over, status):
    assert shared(lib, **over) == status
    assert lib.kap_last_error()


def test_verify_shared_pools_and_empty_batch(lib):
    assert shared(lib, kv_struct(page=32)) == UNS
    assert shared(lib, kv_struct(D=96)) == UNS
    assert shared(lib, kv_struct(num_pages=0)) == BAD
    assert shared(lib, kv_struct(Hq=4096, Hkv=1), w=16) == UNS
    assert shared(lib, kv_struct(Hq=2048, Hkv=1), B=65535, w=16, have=0) == UNS
    assert shared(lib, kv_struct(kv_dtype=K.KAP_DT_FP8_E4M3FN)) == BAD
    assert shared(lib, B=0, groups=0, q=None, lens=None, table=None) == K.KAP_OK
    size = lib.kap_verify_shared_workspace_bytes
    kv = kv_struct()
    assert size(ctypes.byref(kv), 0, 5, 1024, 0) == size(ctypes.byref(kv), 4, 17, 1024, 1) == 0
    assert 0 < size(ctypes.byref(kv), 4, 5, 1024, 1) <= size(ctypes.byref(kv), 8, 5, 1024, 2)
