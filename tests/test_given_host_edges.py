"""Host-side checks of 4-bit vocabulary matrices of local heads, and of the products' self test (no GPU needed)."""
import ctypes
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dels():
    import paper_2607_07409_gb300 as m
    if not os.path.exists(m.library_path()):
        from paper_2607_07409_gb300 import build
        build.build()
    m.lib()
    return m


def head(dels, vocab=8192, **w4):
    h = dels.LocalHead()
    h.kind, h.wdtype, h.d_rank, h.emb, h.w_vocab = dels.DELS_HEAD_MARKOV, dels.DELS_BF16, 64, 4096, vocab
    if w4:
        h.w_vocab4 = ctypes.pointer(dels.W4(w4.get("data", 4096), w4.get("V", 1024), w4.get("K", 64), 32, 0))
    return h


def draft(dels, h, V=1024):
    return dels.lib().dels_draft_block(ctypes.byref(h), 16, 1, 16, 0.3, 0.3, 2, 2, V, 16, 16, None, None, 0, None)


# A head as callers filled it before it had w_vocab4: what lies behind its w_vocab is not the library's to follow.
OLDER = """
import ctypes, paper_2607_07409_gb300 as dels
h = dels.LocalHead()
h.kind, h.wdtype, h.d_rank, h.emb, h.w_vocab = dels.DELS_HEAD_MARKOV, dels.DELS_BF16, 64, 4096, 8192
h.w_vocab4 = ctypes.cast(ctypes.c_void_p(24), type(h.w_vocab4))
L = dels.lib()
L.dels_draft_workspace_bytes(ctypes.byref(h), 2, 2, 1024)
L.dels_draft_state_bytes(ctypes.byref(h), 2, 2)
assert L.dels_draft_block(ctypes.byref(h), 16, 1, 16, 0.3, 0.3, 2, 2, 1024, 16, 16, None, None, 0, None) < 0
w = (ctypes.c_float * 2)(0.3, 0.3)
a = ctypes.cast(w, ctypes.c_void_p)
assert L.dels_verify_block_sampled(ctypes.byref(h), 16, 16, 16, 16, 1, 16, a, a, 16, 1, 2, 2, 1024, 1, 2, 16, 16, None,
                                   4096, 8, None) < 0
print("kept to w_vocab")
"""


def test_a_head_with_w_vocab_is_read_no_further(dels):
    r = subprocess.run([sys.executable, "-c", OLDER], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and "kept to w_vocab" in r.stdout, (r.returncode, r.stderr[-300:])


@pytest.mark.parametrize("code,vocab,w4", [
    (-1, None, {}), (-1, None, dict(data=None)), (-2, None, dict(V=1032)), (-2, None, dict(K=96)),
    (-4, None, dict(data=4104)),
    (-5, None, dict(data=4096)), (-5, 8192, dict(V=1032, K=96, data=1)),       # (as far as the workspace: it is not given)
])
def test_heads_with_a_4_bit_matrix(dels, code, vocab, w4):
    assert draft(dels, head(dels, vocab, **w4)) == code


@pytest.mark.parametrize("code,args", [
    (-2, (4, 1, 2, 128, 32, 4096, 1 << 20)), (-2, (0, 0, 2, 128, 32, 4096, 1 << 20)), (-2, (0, 3, 2, 128, 32, 4096, 1 << 20)),
    (-2, (0, 1, 0, 128, 32, 4096, 1 << 20)), (-2, (0, 1, 129, 128, 32, 4096, 1 << 20)), (-2, (0, 1, 2, 12, 32, 4096, 1 << 20)),
    (-2, (0, 1, 2, 128, 0, 4096, 1 << 20)), (-5, (0, 1, 2, 128, 32, None, 1 << 20)), (-5, (0, 1, 2, 128, 32, 4096, 256)),
    (-4, (0, 1, 2, 128, 32, 4104, 1 << 20)),
])
def test_the_self_test_of_4_bit_products_refuses(dels, code, args):
    assert dels.lib().dels_selftest_w4_timeout(*args, None) == code
