"""Operators of a served verification step without a GPU: what the host refuses before anything is launched, and pins of the
plain references that the GPU tests compare with."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import serve_oracle as SO
from paper_2603_12617_amd import binding as B

ONE = 256                                  # any non-null, aligned address: refused before it is touched
EINVAL, EUNSUPPORTED, ENOMEM = -1, -2, -4


def _step(**over):
    f = dict(B=2, page=16, width=4, table_stride=4, pool=8, tokens=3)
    f.update({n: ONE + 64 * i for i, n in enumerate(("pages", "length", "accepted", "add", "nfree", "table", "free", "pages_out", "length_out",
                                                     "kv_out", "nfree_out", "cu_out", "slot_out", "pos_out"))})
    f.update(over)
    return B.SdPageStep(**f)


@pytest.mark.parametrize("over,rc", [
    (dict(B=0), EINVAL), (dict(page=0), EINVAL), (dict(width=0), EINVAL), (dict(table_stride=3), EINVAL), (dict(pool=0), EINVAL), (dict(tokens=-1), EINVAL),
    (dict(pages=None), EINVAL), (dict(nfree=None), EINVAL), (dict(table=None), EINVAL), (dict(slot_out=None), EINVAL), (dict(cu_out=None), EINVAL),
    (dict(add=258), EINVAL), (dict(pos_out=257), EINVAL), (dict(pages_out=ONE), EINVAL), (dict(nfree_out=ONE + 64 * 4), EINVAL),
    (dict(B=4097), EUNSUPPORTED), (dict(pool=1 << 31), EUNSUPPORTED), (dict(page=1 << 28, pool=9), EUNSUPPORTED),
    (dict(width=1 << 27, table_stride=1 << 27, page=16), EUNSUPPORTED), (dict(B=4096, width=1 << 19, table_stride=1 << 19), EUNSUPPORTED)])
def test_page_steps_that_are_refused(over, rc):
    assert B.lib().sd_pages(C.byref(_step(**over)), None) == rc
    assert B.lib().sd_pages(None, None) == EINVAL


def _cache(**over):
    f = dict(k=ONE, v=ONE, pages=4, page=16, heads=2, D=64, k_page_stride=2048, k_tok_stride=128, k_head_stride=64, v_page_stride=2048, v_tok_stride=128,
             v_head_stride=64, dtype=1)
    f.update(over)
    return B.SdCache(**f)


@pytest.mark.parametrize("over,call,rc", [
    (dict(k=None), {}, EINVAL), (dict(pages=0), {}, EINVAL), (dict(dtype=3), {}, EINVAL), (dict(k=257), {}, EINVAL), (dict(v_tok_stride=-8), {}, EINVAL),
    (dict(page=1 << 30), {}, EUNSUPPORTED), ({}, dict(k=None), EINVAL), ({}, dict(slot=None), EINVAL), ({}, dict(slot=258), EINVAL), ({}, dict(tokens=-1), EINVAL),
    ({}, dict(tokens=1 << 31), EUNSUPPORTED), ({}, dict(ks=-1), EINVAL)])
def test_cache_writes_that_are_refused(over, call, rc):
    a = dict(k=ONE, ks=128, slot=ONE, tokens=3)
    a.update(call)
    c = _cache(**over)
    assert B.lib().sd_cache_store(C.byref(c), a["k"], a["ks"], 64, ONE, 128, 64, a["slot"], a["tokens"], None) == rc
    assert B.lib().sd_cache_store(None, ONE, 128, 64, ONE, 128, 64, ONE, 3, None) == EINVAL


def _attention(cache=None, **over):
    f = dict(cache=_cache(**(cache or {})), B=2, tokens=6, Hq=4, width=4, table_stride=4, q=ONE, q_tok_stride=256, q_head_stride=64, out=ONE, out_tok_stride=256,
             out_head_stride=64, lse=None, cu=ONE, kv=ONE, table=ONE, window=0, scale=0.125)
    f.update(over)
    return B.SdAttention(**f)


@pytest.mark.parametrize("cache,over,rc", [
    ({}, dict(B=0), EINVAL), ({}, dict(tokens=-1), EINVAL), ({}, dict(Hq=3), EINVAL), ({}, dict(Hq=0), EINVAL), ({}, dict(width=0), EINVAL),
    ({}, dict(table_stride=2), EINVAL), ({}, dict(window=-1), EINVAL), ({}, dict(scale=0.0), EINVAL), ({}, dict(scale=-1.0), EINVAL),
    ({}, dict(scale=math.nan), EINVAL), ({}, dict(scale=math.inf), EINVAL), ({}, dict(q_tok_stride=100), EINVAL), ({}, dict(out_head_stride=-64), EINVAL),
    (dict(k_tok_stride=4), {}, EINVAL), (dict(dtype=7), {}, EINVAL), (dict(D=0), {}, EINVAL), (dict(page=0), {}, EINVAL),
    (dict(dtype=0), {}, EUNSUPPORTED), (dict(D=60), {}, EUNSUPPORTED), (dict(D=264), {}, EUNSUPPORTED), ({}, dict(B=4097), EUNSUPPORTED),
    (dict(page=1 << 30), {}, EUNSUPPORTED), ({}, dict(width=1 << 28, table_stride=1 << 28), EUNSUPPORTED), ({}, dict(tokens=1 << 30), EUNSUPPORTED)])
def test_attention_sizes_that_are_refused(cache, over, rc):
    a = _attention(cache, **over)
    assert B.lib().sd_attend_workspace_bytes(C.byref(a)) == 0
    assert B.lib().sd_attend(C.byref(a), ONE, 1 << 40, None) == rc


@pytest.mark.parametrize("cache,over", [(dict(k=None), {}), (dict(v=264), {}), ({}, dict(q=None)), ({}, dict(q=264)), ({}, dict(out=None)), ({}, dict(lse=258)),
                                        ({}, dict(cu=None)), ({}, dict(kv=None)), ({}, dict(table=None)), ({}, dict(table=258))])
def test_attention_pointers_that_are_refused(cache, over):
    a = _attention(cache, **over)
    need = B.lib().sd_attend_workspace_bytes(C.byref(a))
    assert need > 0
    assert B.lib().sd_attend(C.byref(a), ONE, need, None) == EINVAL


def test_attention_workspace():
    a = _attention()
    need = B.lib().sd_attend_workspace_bytes(C.byref(a))
    assert B.lib().sd_attend(C.byref(a), ONE, need - 1, None) == ENOMEM
    assert B.lib().sd_attend(C.byref(a), None, need, None) == EINVAL
    assert B.lib().sd_attend(C.byref(a), 264, need, None) == EINVAL
    assert B.lib().sd_attend(None, ONE, need, None) == EINVAL and B.lib().sd_attend_workspace_bytes(None) == 0
    none = _attention(tokens=0, q=None, out=None)             # no tokens: nothing to do
    assert B.lib().sd_attend(C.byref(none), ONE, B.lib().sd_attend_workspace_bytes(C.byref(none)), None) == 0


def _verify(**over):
    f = dict(B=2, rows=6, V=1000, dtype=1, p=ONE, p_stride=1000, q=ONE, q_stride=1000, tok=ONE, r=ONE, noise=ONE, noise_stride=1000, tau=ONE, cu=ONE)
    f.update(over)
    return B.SdLogits(**f)


@pytest.mark.parametrize("over,rc", [
    (dict(B=0), EINVAL), (dict(V=0), EINVAL), (dict(rows=1), EINVAL), (dict(p_stride=999), EINVAL), (dict(q_stride=999), EINVAL), (dict(noise_stride=10), EINVAL),
    (dict(dtype=5), EINVAL), (dict(V=262145, p_stride=262145, q_stride=262145, noise_stride=262145), EUNSUPPORTED), (dict(B=4097, rows=5000), EUNSUPPORTED)])
def test_verification_sizes_that_are_refused(over, rc):
    a = _verify(**over)
    assert B.lib().sd_verify_logits_workspace_bytes(C.byref(a)) == 0
    assert B.lib().sd_verify_logits(C.byref(a), ONE, ONE, ONE, 1 << 40, None) == rc


def test_verification_pointers_and_workspace():
    L = B.lib()
    need = L.sd_verify_logits_workspace_bytes(C.byref(_verify()))
    assert need > 0
    for over in (dict(p=None), dict(p=257), dict(q=257), dict(tok=None), dict(r=None), dict(r=258), dict(noise=None), dict(tau=None), dict(cu=None), dict(cu=258)):
        assert L.sd_verify_logits(C.byref(_verify(**over)), ONE, ONE, ONE, need, None) == EINVAL, over
    a = _verify()
    assert L.sd_verify_logits(C.byref(a), None, ONE, ONE, need, None) == EINVAL
    assert L.sd_verify_logits(C.byref(a), ONE, 258, ONE, need, None) == EINVAL
    assert L.sd_verify_logits(C.byref(a), ONE, ONE, None, need, None) == EINVAL
    assert L.sd_verify_logits(C.byref(a), ONE, ONE, ONE, need - 1, None) == ENOMEM
    assert L.sd_verify_logits(None, ONE, ONE, ONE, need, None) == EINVAL
    assert L.sd_strerror(ENOMEM) not in (b"ok", b"unknown status")


# ---------------------------------------------------------------- pins of the references ----
def test_pages_by_hand():
    """Two requests, pages of 4 tokens, pages 6 and 7 free (7 on top).  Request 0 had 5 tokens and 3 pages for its drafts (2, 0, 5), one
    draft was accepted: 7 tokens are valid, 1 new one ends at 8: two pages, page 5 goes back.  Request 1 holds page 4 with 3 tokens (0 accepted: 4)
    and gets 6 new ones: 10 tokens, two more pages: 5 (pushed last) and 7."""
    got = SO.pages([3, 1], [5, 3], [1, 6], np.array([[2, 0, 5], [4, -1, -1]]), np.array([6, 7, -1, -1]), 2, 4, accepted=[1, 0])
    assert got["length"].tolist() == [7, 4] and got["kv"].tolist() == [8, 10] and got["pages"].tolist() == [2, 3]
    assert got["table"][1].tolist() == [4, 5, 7] and got["nfree"].tolist() == [1] and got["free"][0] == 6
    assert got["cu"].tolist() == [0, 1, 7] and got["pos"].tolist() == [7, 4, 5, 6, 7, 8, 9]
    assert got["slot"].tolist() == [0 * 4 + 3, 20, 21, 22, 23, 28, 29]


def test_pages_that_are_missing():
    """Three requests want 1, 3 and 1 pages of 3: the second finds too few, and the third behind it gets none either."""
    got = SO.pages([0, 0, 0], [0, 0, 0], [2, 12, 1], np.full((3, 4), -1), np.array([8, 9, 3]), 3, 4)
    assert got["pages"].tolist() == [1, 0, 0] and got["kv"].tolist() == [2, 0, 0] and got["nfree"].tolist() == [2]
    assert got["slot"].tolist() == [12, 13] + [-1] * 13


def test_attention_by_hand():
    """Equal scores average the visible values; one dominant score picks its value; a window hides the first."""
    k = np.zeros((2, 2, 1, 8)); v = np.zeros((2, 2, 1, 8))
    v[1, 0, 0], v[1, 1, 0], v[0, 0, 0] = 1.0, 2.0, 6.0                # keys 0, 1, 2 on pages 1, 1, 0
    table, cu, kv = [[1, 0]], [0, 2], [3]
    out, lse, _, _ = SO.attend(np.ones((2, 1, 8)), k, v, cu, kv, table, 1.0)
    assert np.allclose(out[:, 0, 0], [1.5, 3.0]) and np.allclose(lse[:, 0], np.log([2, 3]))
    out, _, _, _ = SO.attend(np.ones((2, 1, 8)), k, v, cu, kv, table, 1.0, window=2)
    assert np.allclose(out[:, 0, 0], [1.5, 4.0])
    k[1, 1, 0] = 10.0
    out, lse, _, _ = SO.attend(np.ones((2, 1, 8)), k, v, cu, kv, table, 1.0)
    assert np.allclose(out[:, 0, 0], 2.0) and np.allclose(lse, 80.0)
    out, lse, _, _ = SO.attend(np.ones((2, 1, 8)), k, v, cu, [1], table, 1.0)
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all() and np.allclose(out[1], 1.0)


def test_verification_by_hand():
    """V = 3, probabilities (.5, .25, .25) and (.25, .5, .25) as logits: draft 1 has P/Q = 1/2."""
    p = np.log(np.array([[0.5, 0.25, 0.25], [0.2, 0.2, 0.6]])); q = np.log(np.array([[0.25, 0.5, 0.25]]))
    noise, one = np.array([[1.0, 1e-9, 1.0]]), np.ones(1)
    assert [int(x[0]) for x in SO.verify_logits(p, q, [1], [0.49], noise, one, [0, 2])[:2]] == [1, 1]          # accepted; the race for row 1 goes to token 1
    assert [int(x[0]) for x in SO.verify_logits(p, q, [1], [0.51], noise, one, [0, 2])[:2]] == [0, 0]          # rejected; the residual is token 0 alone
    assert [int(x[0]) for x in SO.verify_logits(p, None, [1], [0.24], noise, one, [0, 2])[:2]] == [1, 1]       # without a distribution: P(1) = 1/4
    assert [int(x[0]) for x in SO.verify_logits(p, None, [0], [0.51], noise, one, [0, 2])[:2]] == [0, 1]       # the draft cannot come again
    assert [int(x[0]) for x in SO.verify_logits(p, q, [1], [0.0], noise, 0 * one, [0, 2])[:2]] == [0, 0]       # greedy
    assert [int(x[0]) for x in SO.verify_logits(p, q, [0], [0.9], noise, 0 * one, [0, 2])[:2]] == [1, 2]
