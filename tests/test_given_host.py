"""Host-side checks of the 4-bit products, the probabilities of rows and the verification from given numbers
(no GPU needed): bad arguments are refused before a device is touched."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def dels():
    import paper_2607_07409_gb300 as m
    if not os.path.exists(m.library_path()):
        from paper_2607_07409_gb300 import build
        build.build()
    m.lib()
    return m


WS = 1 << 12   # an aligned address that is never read on the host


def ref(struct, **kw):
    for k, v in kw.items():
        setattr(struct, k, v)
    return ctypes.byref(struct)


# ---------------------------------------------------------------- 4-bit matrices

def test_w4_bytes(dels):
    # for 128 rows and 128 inputs: codes, 256 bytes of scales and 64 of zero points a group
    assert dels.dels_w4_bytes(32, 128, 128, False) == 8192 + 256
    assert dels.dels_w4_bytes(129, 128, 32, True) == 2 * (8192 + 4 * 320)
    assert dels.dels_w4_bytes(1, 1, 64, True) == 8192 + 2 * 320
    assert dels.dels_w4_bytes(64, 1000, 64, False) == 8 * (8192 + 2 * 256)
    for V, K, G in [(0, 128, 32), (8, 0, 32), (8, 128, 16), (8, 128, 48), (8, 128, 256), ((1 << 27) + 1, 8, 32),
                    (8, 65537, 32), (-1, 8, 32)]:
        assert dels.dels_w4_bytes(V, K, G, False) == 0


def pack(dels, codes=64, scales=64, zeros=None, V=40, K=100, group=32, packed=4096, nbytes=1 << 20, ws=WS, n=256):
    return dels.lib().dels_w4_pack(codes, scales, zeros, V, K, group, packed, nbytes, ws, n, None)


@pytest.mark.parametrize("code,kw", [
    (-2, dict(V=0)), (-2, dict(K=0)), (-2, dict(group=48)), (-2, dict(K=65537)),
    (-1, dict(codes=None)), (-1, dict(scales=None)), (-1, dict(packed=None)),
    (-5, dict(ws=None)), (-5, dict(n=255)), (-5, dict(nbytes=4 * 2048 + 4 * 256 - 1)),
    (-5, dict(zeros=64, nbytes=4 * 2048 + 4 * 320 - 1)),
    (-4, dict(packed=4104)), (-4, dict(scales=65)), (-4, dict(ws=WS + 8)),
])
def test_pack_refuses(dels, code, kw):
    assert pack(dels, **kw) == code


def project(dels, w=None, x=64, xt=1, xs=0, B=2, out=64, ot=0, os_=0, ws=WS, n=256, **kw):
    m = dels.W4(4096, 40, 100, 32, 0)
    return dels.lib().dels_w4_project(ref(m, **kw), x, xt, xs, B, out, ot, os_, ws, n, None)


@pytest.mark.parametrize("code,kw", [
    (-1, dict(data=None)), (-2, dict(V=0)), (-2, dict(K=0)), (-2, dict(group=33)), (-4, dict(data=4104)),
    (-3, dict(xt=2)), (-3, dict(ot=7)), (-2, dict(B=-1)), (-2, dict(B=65536)), (-2, dict(xs=99)), (-2, dict(os_=39)),
    (-5, dict(ws=None)), (-5, dict(n=255)), (-1, dict(x=None)), (-1, dict(out=None)),
    (-4, dict(x=65)), (-4, dict(x=66, xt=0)), (-4, dict(out=66)), (-4, dict(out=65, ot=1)), (-4, dict(ws=WS + 8)),
    (0, dict(B=0)), (0, dict(B=0, x=None, out=None)),
])
def test_project_refuses(dels, code, kw):
    assert project(dels, **kw) == code


def test_pack_w4_refuses(dels):
    codes = torch.zeros(8, 64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        dels.pack_w4(codes, torch.zeros(8, 2, dtype=torch.bfloat16), group=32)
    with pytest.raises(ValueError, match=r"\[V, K\]"):
        dels.pack_w4(codes[0], None, group=32)


# ---------------------------------------------------------------- probabilities

def probs(dels, R=2, V=8, out=64, ot=0, os_=0, ws=WS, n=256, **kw):
    x = dels.Rows()
    x.long_logits, x.dtype, x.temperature = 4096, 0, 1.0
    return dels.lib().dels_row_probs(ref(x, **kw), R, V, out, ot, os_, ws, n, None)


@pytest.mark.parametrize("code,kw", [
    (-3, dict(dtype=5)), (-3, dict(ot=2)), (-2, dict(R=-1)), (-2, dict(V=0)), (-2, dict(V=(1 << 30) + 1)),
    (-2, dict(temperature=0.0)), (-2, dict(temperature=float("nan"))), (-2, dict(long_stride=7)), (-2, dict(os_=7)),
    (-1, dict(long_logits=None)), (-1, dict(out=None)), (-4, dict(out=66)), (-4, dict(out=65, ot=1)),
    (-4, dict(long_logits=4098)), (-5, dict(ws=None)), (-5, dict(n=8)), (-4, dict(ws=WS + 8)),
    (-2, dict(alpha=64)), (0, dict(R=0)), (0, dict(R=0, out=None, long_logits=None)),
])
def test_row_probs_refuses(dels, code, kw):
    assert probs(dels, **kw) == code


def test_row_probs_size(dels):
    assert dels.dels_row_probs_workspace_bytes(3, 100) >= 4
    assert dels.dels_row_probs_workspace_bytes(-1, 100) == 0 and dels.dels_row_probs_workspace_bytes(1, 0) == 0
    assert dels.dels_row_probs_workspace_bytes(1, (1 << 30) + 1) == 0


# ---------------------------------------------------------------- verification

def verify(dels, tokens=64, uniforms=64, lengths=None, B=2, n=4, V=8, acc=64, bonus=64, ws=WS, nbytes=256, target=True,
           draft=True, **kw):
    p, q = dels.Probs(4096, 0, 0, 0), dels.Probs(8192, 1, 0, 0)
    for k, v in kw.items():
        setattr(p if k[0] == "p" else q, k[2:], v)
    return dels.lib().dels_verify_given(tokens, ctypes.byref(p) if target else None,
                                        ctypes.byref(q) if draft else None, uniforms, lengths, B, n, V, acc, bonus, ws,
                                        nbytes, None)


@pytest.mark.parametrize("code,kw", [
    (-2, dict(B=-1)), (-2, dict(B=(1 << 20) + 1)), (-2, dict(n=-1)), (-2, dict(n=1025)), (-2, dict(V=0)),
    (-2, dict(V=(1 << 30) + 1)), (-3, dict(p_dtype=2)), (-3, dict(q_dtype=-1)),
    (-2, dict(p_row_stride=7)), (-2, dict(q_row_stride=7)), (-2, dict(p_batch_stride=5 * 8 - 1)),
    (-2, dict(q_batch_stride=4 * 8 - 1)), (-2, dict(p_row_stride=16, p_batch_stride=4 * 16 + 7)),
    (-4, dict(p_data=4098)), (-4, dict(q_data=8193)), (-4, dict(tokens=66)), (-4, dict(uniforms=66)),
    (-4, dict(lengths=66)), (-4, dict(acc=66)), (-4, dict(bonus=66)), (-4, dict(ws=WS + 8)),
    (-1, dict(target=False)), (-1, dict(p_data=None)), (-1, dict(q_data=None)), (-1, dict(tokens=None)),
    (-1, dict(uniforms=None)), (-1, dict(acc=None)), (-1, dict(bonus=None)), (-5, dict(ws=None)), (-5, dict(nbytes=8)),
    (0, dict(B=0)), (0, dict(B=0, p_data=None, tokens=None)),
])
def test_verify_given_refuses(dels, code, kw):
    assert verify(dels, **kw) == code


def test_verify_given_size(dels):
    assert dels.dels_verify_given_workspace_bytes(3, 0, 100) >= 4
    for args in [(-1, 1, 8), (1, -1, 8), (1, 1, 0), (1, 1025, 8), ((1 << 20) + 1, 1, 8)]:
        assert dels.dels_verify_given_workspace_bytes(*args) == 0


def test_status_string(dels):
    assert "out of range" in dels.dels_status_string(dels.DELS_STATUS_BAD_VALUE)
