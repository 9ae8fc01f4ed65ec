"""The operators of a served verification step against plain references: whole numbers exactly, attention to bounds
that follow from its roundings, verified tokens exactly wherever the reference says that no decision was within
float32 rounding of its opposite."""
import numpy as np
import pytest

from oracle import serve_oracle as SO
from paper_2603_12617_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}            # half a unit in the last place, relative (8 and 11 bits of significand)


def _torch():
    import torch
    return torch


def _dt(name):
    torch = _torch()
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def _i32(v):
    return _torch().tensor(np.asarray(v, np.int32), dtype=_torch().int32, device=DEV)


# ------------------------------------------------------------------ block tables ----
def _run_pages(st, page, accepted=None, tokens=None, stream=None):
    torch = _torch()
    Bn = len(st["pages"])
    T = int(np.sum(st["add"])) if tokens is None else tokens
    t = {k: _i32(v) for k, v in st.items()}
    out = {k: torch.full((n,), -77, dtype=torch.int32, device=DEV)
           for k, n in (("pages", Bn), ("length", Bn), ("kv", Bn), ("nfree", 1), ("cu", Bn + 1), ("slot", T), ("pos", T))}
    B.sd_pages(t["pages"], t["length"], t["add"], t["table"], t["free"], t["nfree"], page, out["pages"], out["length"], out["kv"], out["nfree"],
               out["cu"], out["slot"], out["pos"], accepted=None if accepted is None else _i32(accepted), stream=stream)
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in out.items()}
    got["table"], got["free"] = t["table"].cpu().numpy(), t["free"].cpu().numpy()
    return got


def _pages_state(rng, Bn, page, width, pool_extra, len_max, add, held_extra=0):
    length = rng.integers(0, len_max + 1, Bn)
    held = np.minimum(-(-length // page) + rng.integers(0, held_extra + 1, Bn), width)
    length = np.minimum(length, held * page)
    total = int(held.sum())
    ids = rng.permutation(total + pool_extra)
    table = np.full((Bn, width), -5, np.int32)
    k = 0
    for b in range(Bn):
        table[b, :held[b]] = ids[k:k + held[b]]
        k += held[b]
    free = np.full(total + pool_extra, -9, np.int32)
    free[:pool_extra] = ids[k:]
    return dict(pages=held, length=length, add=np.broadcast_to(add, Bn).copy() if np.ndim(add) == 0 else add, table=table, free=free, nfree=np.array([pool_extra]))


def _same_pages(got, want):
    for k in want:
        assert np.array_equal(got[k], want[k]), (k, np.nonzero(got[k] != want[k])[0][:8])


@pytest.mark.parametrize("Bn,page,width,extra,len_max,add", [
    (1, 16, 8, 4, 100, 1), (1, 1, 40, 20, 20, 7), (64, 16, 300, 500, 4000, 5), (65, 24, 40, 300, 700, 9), (1000, 128, 20, 4000, 2000, 300),
    (4096, 16, 40, 9000, 300, 3), (3, 1000, 5, 9, 3000, 0), (257, 7, 64, 1000, 200, 13)])
@pytest.mark.parametrize("step", [False, True])
def test_tables_of_a_step(Bn, page, width, extra, len_max, add, step):
    rng = np.random.default_rng(Bn * 31 + page)
    st = _pages_state(rng, Bn, page, width, extra, min(len_max, width * page), rng.integers(0, add + 1, Bn), held_extra=2)
    acc = rng.integers(0, 6, Bn) if step else None
    print("case", Bn, page, step, flush=True)
    _same_pages(_run_pages(st, page, acc), SO.pages(accepted=acc, page=page, **{**st, "nfree": int(st["nfree"][0])}))


def test_tables_finished_refused_and_repeated():
    rng = np.random.default_rng(5)
    st = _pages_state(rng, 40, 16, 12, 6, 150, rng.integers(0, 60, 40), held_extra=1)
    st["length"][[3, 17]] = 0
    st["add"][[3, 17]] = 0                                   # finished: all pages go back
    st["add"][8] = 16 * 12                                   # too long for the table
    want = SO.pages(page=16, **{**st, "nfree": 6})
    got = _run_pages(st, 16)
    _same_pages(got, want)
    served = want["kv"] == want["length"] + st["add"]
    assert not served.all() and served.any() and want["pages"][3] == 0    # the pool runs out on the way
    # what a call writes it does not read: the same inputs give the same again
    st2 = dict(st, table=got["table"], free=got["free"])
    _same_pages(_run_pages(st2, 16), want)
    # fewer token entries than tokens: the rest is not written
    few = _run_pages(st, 16, tokens=37)
    assert np.array_equal(few["slot"], want["slot"][:37]) and np.array_equal(few["cu"], want["cu"])


@pytest.mark.parametrize("Bn,extra", [(1, 3), (70, 5), (300, 4096)])
def test_tables_of_a_padded_step(Bn, extra):
    """More token entries than tokens: the rest has no slot."""
    rng = np.random.default_rng(Bn)
    st = _pages_state(rng, Bn, 16, 30, 2000, 200, rng.integers(0, 40, Bn))
    T = int(st["add"].sum())
    got, want = _run_pages(st, 16, tokens=T + extra), SO.pages(page=16, **{**st, "nfree": 2000})
    assert np.array_equal(got["slot"][:T], want["slot"]) and np.array_equal(got["pos"][:T], want["pos"])
    assert (got["slot"][T:] == -1).all() and (got["pos"][T:] == -1).all()


def test_tables_clamp_what_the_host_cannot_see():
    """Lengths, counts and stack heights out of range give some result, inside the arrays."""
    rng = np.random.default_rng(6)
    st = _pages_state(rng, 9, 16, 8, 20, 100, 4)
    st["pages"][:4] = [-3, 9, 1 << 30, 8]
    st["length"][:4] = [1 << 30, -7, 0x7fffffff, 5]
    st["add"][4:6] = [-2, 0x7fffffff]
    st["nfree"] = np.array([1 << 20])
    got = _run_pages(st, 16, tokens=50)
    assert (got["pages"] >= 0).all() and (got["pages"] <= 8).all() and 0 <= got["nfree"][0] <= len(st["free"])


# ------------------------------------------------------------------- cache writes ----
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,heads,D,page,first,odd", [
    (1, 8, 128, 16, False, 0), (160, 8, 128, 16, True, 0), (333, 3, 80, 24, False, 0), (77, 1, 64, 1, True, 0), (50, 5, 40, 7, False, 3), (3000, 2, 256, 64, True, 0)])
def test_cache_writes(dtype, T, heads, D, page, first, odd):
    torch = _torch()
    g = torch.Generator(device=DEV).manual_seed(T + D)
    pages = -(-T // page) + 3
    shape = (pages, heads, page, D + odd) if first else (pages, page, heads, D + odd)
    caches = [torch.randn(shape, generator=g, device=DEV).to(_dt(dtype)) for _ in range(2)]
    views = [(c.transpose(1, 2) if first else c)[..., :D] for c in caches]
    new = torch.randn((T, 2 * heads, D + odd), generator=g, device=DEV).to(_dt(dtype))[..., :D]
    k, v = new[:, :heads], new[:, heads:]
    slot = torch.randperm(pages * page, generator=g, device=DEV)[:T].to(torch.int32)
    slot[::5] = -1
    if T > 7:
        slot[6], slot[7] = pages * page, 0x7fffffff
    want = [c.clone() for c in views]
    for i, s in enumerate(slot.tolist()):
        if 0 <= s < pages * page:
            want[0][s // page, s % page] = k[i]
            want[1][s // page, s % page] = v[i]
    B.sd_cache_store(k, v, slot, views[0], views[1])
    torch.cuda.synchronize()
    assert torch.equal(views[0], want[0]) and torch.equal(views[1], want[1])
    B.sd_cache_store(k[:0], v[:0], slot[:0], views[0], views[1])                # no tokens: nothing


# ---------------------------------------------------------------------- attention ----
class _Batch:
    """A batch with its cache: unused slots of the pages, and whatever else no row sees, hold NaN."""

    def __init__(self, new, kv, Hq, Hkv, D, page, dtype, window=0, heads_first=False, seed=0, q_scale=2.0, spare=3):
        torch = _torch()
        self.new, self.kv, self.window, self.dtype = new, kv, window, dtype
        g = torch.Generator(device="cpu").manual_seed(seed + 1)
        dt = _dt(dtype)
        held = [-(-n // page) for n in kv]
        pool, width = sum(held) + spare, max(held + [1]) + 2
        order = torch.randperm(pool, generator=g).tolist()
        table = np.full((len(kv), width), 1 << 30, np.int32)          # (entries past the held pages are never used)
        k = 0
        for b, h in enumerate(held):
            table[b, :h] = order[k:k + h]
            k += h
        shape = (pool, Hkv, page, D) if heads_first else (pool, page, Hkv, D)
        kc, vc = torch.full(shape, float("nan")).to(dt), torch.full(shape, float("nan")).to(dt)
        self.k, self.v = (c.transpose(1, 2) if heads_first else c for c in (kc, vc))
        for b, n in enumerate(kv):
            lo = max(0, n - new[b] - window + 1) if window else 0
            j = torch.arange(lo, n)
            at = torch.tensor(table[b])[j // page].long()
            self.k[at, j % page] = torch.randn((len(j), Hkv, D), generator=g).to(dt)
            self.v[at, j % page] = torch.randn((len(j), Hkv, D), generator=g).to(dt)
        T = sum(new)
        # (heads of queries inside a longer projection)
        self.wide_q = (q_scale * torch.randn((T, Hq + 2, D), generator=g)).to(dt)
        self.q = self.wide_q[:, 1:Hq + 1]
        self.table, self.cu = table, np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.scale = D ** -0.5

    def gpu(self, lse=True, stream=None):
        torch = _torch()
        q, k, v = self.wide_q.to(DEV)[:, 1:self.q.shape[1] + 1], self.k.to(DEV), self.v.to(DEV)
        table, cu, kv = _i32(self.table), _i32(self.cu), _i32(self.kv)
        T, Hq, D = q.shape
        out = torch.full((T, Hq, D), -7.0, dtype=q.dtype, device=DEV)
        l = torch.full((T, Hq), -7.0, device=DEV) if lse else None
        ws = torch.full((B.sd_attend_workspace_bytes(q, k, table),), 0xff, dtype=torch.uint8, device=DEV)    # (NaN)
        torch.cuda.synchronize()
        B.sd_attend(q, k, v, cu, kv, table, out, self.scale, lse=l, window=self.window, ws=ws, stream=stream)
        torch.cuda.synchronize()
        return out, l

    def check(self, **kw):
        out, lse = self.gpu(**kw)
        host = lambda c: c.double().numpy()  # noqa: E731
        want, wlse, size, big = SO.attend(host(self.q), host(self.k), host(self.v), self.cu, self.kv, self.table, self.scale, self.window)
        u, D = UNIT[self.dtype], self.q.shape[2]
        # float32 sums of D products (scores), then of weights: relative 2^-23 a few times per step of 16 elements; a score's
        # absolute error is its weight's relative one.  Weights and results are rounded once each to the type; weights below its
        # range (2^-25 of the largest in float16) vanish.
        es = (D / 16 + 8) * 2.0 ** -23 * (big + 1)
        n = max(list(self.kv) + [1])
        tol = 1.05 * u * (np.abs(want) + size) + (2 * es[..., None] + 2e-6) * size + n * 2.0 ** -25 * 4.0 * (self.dtype == "f16") + 1e-30
        err = np.abs(out.double().cpu().numpy() - want)
        assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
        if lse is not None:
            lse = lse.double().cpu().numpy()
            assert np.array_equal(np.isneginf(lse), np.isneginf(wlse))
            there = ~np.isneginf(wlse)
            assert (np.abs(lse[there] - wlse[there]) <= (es + 2e-6)[there] + 2e-6 * np.abs(wlse[there])).all()
        return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [8, 64, 72, 80, 96, 128, 136, 192, 256])
@pytest.mark.parametrize("new,kv", [([1], [1]), ([5, 1, 0, 3], [300, 1, 0, 77]), ([130, 1, 40], [130, 65, 500])])
def test_attention_head_sizes(dtype, D, new, kv):
    print("case", dtype, D, new, kv, flush=True)
    _Batch(new, kv, 4, 2, D, 16, dtype, seed=D).check()


@pytest.mark.parametrize("page", [1, 7, 16, 24, 64, 200])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (6, 2), (7, 1), (40, 1), (5, 5)])
@pytest.mark.parametrize("many", [False, True])
def test_attention_pages_and_heads(page, Hq, Hkv, many):
    new, kv = ([97, 3, 260], [97, 400, 300]) if many else ([1, 4, 2], [33, 129, 513])
    print("case", page, Hq, Hkv, many, flush=True)
    _Batch(new, kv, Hq, Hkv, 64, page, "bf16", heads_first=page % 2 == 0, seed=page).check()


@pytest.mark.parametrize("window", [1, 5, 64, 100, 1000])
@pytest.mark.parametrize("new,kv", [([1, 4], [1000, 30]), ([200, 31, 64], [700, 40, 64])])
def test_attention_windows(window, new, kv):
    print("case", window, new, kv, flush=True)
    _Batch(new, kv, 4, 2, 128, 16, "f16", window=window, seed=window).check()


@pytest.mark.parametrize("new,kv", [([4], [0]), ([4], [2]), ([300], [260]), ([3, 0, 2], [1, 0, 900]), ([1], [0])])
def test_attention_rows_without_a_key(new, kv):
    b = _Batch(new, kv, 4, 2, 64, 16, "bf16")
    out, lse = b.check()
    first = max(0, new[0] - kv[0])
    assert (out[:first] == 0).all() and np.isneginf(lse[:first]).all()


@pytest.mark.parametrize("new,kv,Hq,Hkv,D", [([1], [5000], 8, 8, 128), ([5, 5], [4097, 20], 8, 1, 64), ([70], [3000], 4, 1, 128), ([2], [2500], 4, 2, 256)])
def test_attention_long_contexts_are_split_and_joined(new, kv, Hq, Hkv, D):
    for dtype in ("bf16", "f16"):
        _Batch(new, kv, Hq, Hkv, D, 32, dtype, seed=3).check()


def test_attention_extreme_scores():
    """Scores far apart: the running maximum moves by thousands, weights vanish."""
    for new, kv in (([3], [700]), ([150], [700])):
        b = _Batch(new, kv, 4, 2, 64, 16, "bf16", q_scale=200.0, seed=9)
        b.check()


def test_attention_masked_keys_of_a_chunk_do_not_matter():
    """A row gives the same bits whatever finite values the later tokens of its chunk hold."""
    b = _Batch([100], [300], 4, 2, 64, 16, "bf16", seed=4)
    out, _ = b.gpu()
    j = _torch().arange(250, 300)
    at = _torch().tensor(b.table[0])[j // 16].long()
    b.k[at, j % 16], b.v[at, j % 16] = 3e4, -3e4
    again, _ = b.gpu()
    assert _torch().equal(out[:50], again[:50]) and not _torch().equal(out[50:], again[50:])


@pytest.mark.parametrize("new,kv", [([3], [40]), ([3], [3000]), ([150], [400])])
def test_attention_numbers_that_are_none_stay_in_sight(new, kv):
    """A query that is no number gives a row that is none, and a key that is none the rows that see it; the other rows keep their bits."""
    torch = _torch()
    b = _Batch(new, kv, 4, 2, 64, 16, "bf16", seed=6)
    clean, clean_lse = b.gpu()
    b.wide_q[1, 2, 7] = float("nan")                                  # token 1, query head 1
    out, lse = b.gpu()
    assert torch.isnan(out[1, 1]).all() and torch.isnan(lse[1, 1])
    keep = torch.ones_like(lse, dtype=torch.bool)
    keep[1, 1] = False
    assert torch.equal(out[keep], clean[keep]) and torch.equal(lse[keep], clean_lse[keep])
    b.wide_q[1, 2, 7] = 0.5
    clean, clean_lse = b.gpu()
    last = kv[0] - 1                                                  # the last key, key head 1: seen by the last row's heads 2 and 3 alone
    b.k[int(b.table[0, last // 16]), last % 16, 1, 3] = float("nan")
    out, lse = b.gpu()
    assert torch.isnan(out[-1, 2:]).all() and torch.isnan(lse[-1, 2:]).all()
    assert torch.equal(out[:-1], clean[:-1]) and torch.equal(out[-1, :2], clean[-1, :2]) and torch.equal(lse[:-1], clean_lse[:-1])


@pytest.mark.parametrize("Bn,most,Hq", [(65, 3, 2), (300, 9, 4), (4096, 1, 1), (130, 70, 1)])
def test_attention_of_many_requests(Bn, most, Hq):
    rng = np.random.default_rng(Bn)
    new = rng.integers(0, most + 1, Bn).tolist()
    kv = [int(n + rng.integers(0, 60)) for n in new]
    _Batch(new, kv, Hq, 1, 64, 16, "f16", seed=Bn).check()


@pytest.mark.parametrize("new,kv,Hq,Hkv,D,window", [
    ([1] * 70, [20000] + [50] * 69, 2, 1, 64, 0), ([1, 0, 2] * 34, [9000 if b == 40 else 30 + b for b in range(102)], 8, 8, 128, 0),
    ([3, 1, 0, 2], [6000, 5000, 4000, 7], 4, 2, 64, 0), ([9] * 5, [700, 5000, 9, 1300, 2500], 8, 1, 128, 0), ([1] * 20, list(range(100, 6100, 300)), 16, 16, 64, 0),
    ([2, 2, 2], [9000, 400, 8000], 4, 2, 64, 3000), ([1] * 300, [40] * 299 + [12000], 2, 2, 256, 0)])
def test_attention_of_contexts_of_very_different_lengths(new, kv, Hq, Hkv, D, window):
    """Keys are split where few requests would leave the chip empty, and where one is far longer than the others."""
    print("case", len(new), max(kv), Hq, Hkv, D, flush=True)
    _Batch(new, kv, Hq, Hkv, D, 16, "bf16", seed=D + len(new), window=window).check()


def test_attention_clamps_what_the_host_cannot_see():
    """Offsets, lengths and page numbers out of range give some result, inside the arrays."""
    torch = _torch()
    for new, kv in (([2, 3, 1], [2500, 100, 900]), ([90, 60, 50], [200, 300, 60])):
        b = _Batch(new, kv, 4, 2, 64, 16, "bf16", seed=5)
        T = sum(new)
        for cu, lengths in (([0, T, 0, T], kv), ([-5, 1 << 30, 7, -1], kv), ([0, 0, 0, 0], kv), (b.cu.tolist(), [-1, 1 << 30, 0x7fffffff])):
            bad = _Batch(new, kv, 4, 2, 64, 16, "bf16", seed=5)
            bad.cu, bad.kv, bad.table = np.array(cu, np.int32), lengths, np.where(bad.table == 1 << 30, -7, bad.table)
            out, _ = bad.gpu()
            assert out.shape[0] == T
        want, _ = b.gpu()
        assert torch.isfinite(want).all()                       # and the next call is not the worse for it
        b.check()


def test_attention_workspace_contents_do_not_matter():
    """Tokens before the first request's have no parts: whatever the workspace holds in their place is not taken for some."""
    torch = _torch()
    for new, kv in (([2, 3], [2500, 100]), ([90, 60], [200, 300])):
        b = _Batch(new, kv, 4, 2, 64, 16, "bf16", seed=5)
        want, _ = b.gpu()
        q, k, v = (x.to(DEV) for x in (b.q, b.k, b.v))
        cu, lengths, table = _i32(b.cu), _i32(b.kv), _i32(b.table)
        cu[0] = 1                                                # (the first request has a token less; its others stand where they did)
        for fill in (0x7f, 0x00, 0x01, 0x80, 0xff):
            out = torch.full(tuple(q.shape), -7.0, dtype=q.dtype, device=DEV)
            ws = torch.full((B.sd_attend_workspace_bytes(q, k, table),), fill, dtype=torch.uint8, device=DEV)
            for _ in range(2):                                   # (and what the last call left there)
                B.sd_attend(q, k, v, cu, lengths, table, out, b.scale, ws=ws)
            torch.cuda.synchronize()
            assert (out[0] == -7).all() and (out[1:] != -7).any(dim=-1).all()
            B.sd_attend(q, k, v, _i32(b.cu), lengths, table, out, b.scale, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            B.sd_attend(q, k, v, cu, lengths, table, out.fill_(-7.0), b.scale, ws=ws)     # (row 0's parts lie there now)
            torch.cuda.synchronize()
            assert (out[0] == -7).all()


def test_attention_of_a_padded_batch():
    """Rows past the last request's are nobody's: they are left alone, the others' are the same."""
    torch = _torch()
    for new, kv in (([2, 3], [2500, 100]), ([90, 60], [200, 300])):
        b = _Batch(new, kv, 4, 2, 64, 16, "bf16", seed=5)
        want, _ = b.gpu()
        extra = torch.ones((11,) + tuple(b.wide_q.shape[1:]), dtype=b.wide_q.dtype)
        b.wide_q = torch.cat([b.wide_q, extra])
        b.q = b.wide_q[:, 1:5]
        out, _ = b.gpu()
        assert torch.equal(out[:sum(new)], want) and (out[sum(new):] == -7).all()


def test_attention_offsets_beyond_32_bits():
    torch = _torch()
    page, Hkv, D = 64, 8, 128
    pages = (1 << 32) // (page * Hkv * D) + 40                       # more than 2^32 elements a side
    k = torch.zeros((pages, page, Hkv, D), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    n = 200
    b = _Batch([3], [n], 16, Hkv, D, page, "bf16", seed=8)
    used = [pages - 1, pages - 17, 0, pages - 5]
    new = torch.randn((n, 2 * Hkv, D), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    slot = _i32([used[j // page] * page + j % page for j in range(n)])
    B.sd_cache_store(new[:, :Hkv], new[:, Hkv:], slot, k, v)
    table = _i32([used + [0, 0]])
    q, out = b.q.to(DEV), torch.empty((3, 16, D), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(B.sd_attend_workspace_bytes(q, k, table), dtype=torch.uint8, device=DEV)
    B.sd_attend(q, k, v, _i32([0, 3]), _i32([n]), table, out, b.scale, ws=ws)
    torch.cuda.synchronize()
    small = torch.full((6, page, Hkv, D), 0.0, dtype=torch.bfloat16, device=DEV)
    ks, vs = small, small.clone()
    B.sd_cache_store(new[:, :Hkv], new[:, Hkv:], _i32(list(range(n))), ks, vs)
    t2, out2 = _i32([[0, 1, 2, 3, 0, 0]]), torch.empty_like(out)
    B.sd_attend(q, ks, vs, _i32([0, 3]), _i32([n]), t2, out2, b.scale, ws=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and float(out.float().abs().sum()) > 0


@pytest.mark.parametrize("D", [96, 192, 128])
@pytest.mark.parametrize("new", [[5, 1], [200, 40]])
def test_attention_reads_nothing_behind_the_cache(D, new):
    """A cache that ends where its memory does (whole blocks of 2 MiB), its last row in use: heads that do not fill their row of LDS too."""
    b = _Batch(new, [64 * 127, 64], 8, 8, D, 64, "bf16", seed=D, spare=0)
    assert b.k.numel() * 2 % (2 << 20) == 0 and b.k.shape[0] - 1 in b.table[:, :127]
    print("case", D, new, flush=True)
    b.check()


def test_attention_repeats_its_bits_and_runs_on_other_streams():
    torch = _torch()
    b = _Batch([5, 33, 1], [900, 400, 2000], 8, 2, 128, 16, "bf16", seed=12)
    first, l1 = b.gpu()
    s = torch.cuda.Stream()
    second, l2 = b.gpu(stream=s)
    third, _ = b.gpu(lse=False)
    assert torch.equal(first, second) and torch.equal(l1, l2) and torch.equal(first, third)


# ------------------------------------------------------------------- verification ----
def _logits(rng, k, V, dtype, draft=True, tau=(0.6, 1.2), greedy=0.0, noise=0.6, pad=0):
    torch = _torch()
    Bn, T = len(k), sum(k) + len(k)
    lp = 2.5 * rng.standard_normal((T, V)).astype(np.float32)
    cu = np.concatenate([[0], np.cumsum([x + 1 for x in k])]).astype(np.int32)
    rows = np.concatenate([np.arange(cu[b], cu[b] + k[b]) for b in range(Bn)]).astype(int)
    lq = lp[rows] + noise * rng.standard_normal((len(rows), V)).astype(np.float32)
    t = rng.uniform(*tau, Bn).astype(np.float32)
    t[rng.permutation(Bn)[:int(greedy * Bn)]] = 0.0
    p = torch.tensor(np.pad(lp, ((0, 0), (0, pad)))).to(_dt(dtype))[:, :V]
    q = torch.tensor(np.pad(lq, ((0, 0), (0, pad)))).to(_dt(dtype))[:, :V] if draft else None
    req = np.repeat(np.arange(Bn), k)
    tq = np.maximum(t[req], 0.25)[:, None]
    tok = np.argmax((lq if draft else lp[rows]) / tq + rng.gumbel(size=lq.shape), axis=1) if len(rows) else np.zeros(0)
    return dict(p=p, q=q, tok=tok.astype(np.int32), r=rng.random(len(rows), dtype=np.float32),
                noise=rng.exponential(size=(Bn, V)).astype(np.float32), tau=t, cu=cu)


def _run_verify(d, stream=None):
    torch = _torch()
    f = lambda a: torch.tensor(a, device=DEV)  # noqa: E731
    p, q = d["p"].to(DEV), None if d["q"] is None else d["q"].to(DEV)
    if d["p"].stride(0) != d["p"].shape[1]:                 # (.to() may have made them whole)
        wide = lambda x: torch.nn.functional.pad(x, (0, d["p"].stride(0) - x.shape[1]))[:, :x.shape[1]]  # noqa: E731
        p, q = wide(p), None if q is None else wide(q)
    Bn = len(d["tau"])
    n, nx = (torch.full((Bn,), -7, dtype=torch.int32, device=DEV) for _ in range(2))
    tau = f(d["tau"])
    ws = torch.full((B.sd_verify_logits_workspace_bytes(p, q, tau),), 0xff, dtype=torch.uint8, device=DEV)
    args = (p, q, f(d["tok"]), f(d["r"]), f(d["noise"]), tau, f(d["cu"]), n, nx, ws)
    torch.cuda.synchronize()
    B.sd_verify_logits(*args, stream=stream)
    torch.cuda.synchronize()
    return n.cpu().numpy(), nx.cpu().numpy()


def _check_verify(d):
    n, nx = _run_verify(d)
    host = lambda x: None if x is None else x.double().numpy()  # noqa: E731
    wn, wx, close = SO.verify_logits(host(d["p"]), host(d["q"]), d["tok"], d["r"], d["noise"], d["tau"], d["cu"])
    # a probability's relative error: (l - max) / tau <= 80 rounded three times (1.5e-5), sums 1e-6; scores add a division
    sure = close > 4e-5
    assert sure.mean() > 0.9 or len(sure) < 20
    assert np.array_equal(n[sure], wn[sure]), (n, wn)
    assert np.array_equal(nx[sure], wx[sure]), (nx, wx, close)
    return n, nx


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k,V", [([4] * 8, 1000), ([0], 7), ([1], 1), ([0, 3, 1, 8, 0], 4099), ([1, 0, 2] * 50, 700), ([2] * 30, 8192), ([3] * 5, 8193), ([5, 70], 300), ([2, 2], 50257),
                                 ([1], 262144)])
@pytest.mark.parametrize("draft", [True, False])
def test_verified_tokens(dtype, k, V, draft):
    rng = np.random.default_rng(V + len(k))
    print("case", dtype, k[:6], V, draft, flush=True)
    _check_verify(_logits(rng, k, V, dtype, draft, greedy=0.3 if len(k) > 2 else 0.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [1, 2, 7, 12, 20, 700, 1003, 8191, 8198])
@pytest.mark.parametrize("greedy", [False, True])
def test_every_place_of_a_row_is_read(dtype, V, greedy):
    """One logit far above the others, at each of the first and last places of a row of any length."""
    torch = _torch()
    xs = sorted(set(range(min(V, 10))) | set(range(max(0, V - 18), V)))
    p = torch.full((len(xs), V), -5.0)
    p[range(len(xs)), xs] = 30.0
    none = np.zeros(0, np.int32)
    d = dict(p=p.to(_dt(dtype)), q=None, tok=none, r=none.astype(np.float32), noise=np.ones((len(xs), V), np.float32),
             tau=np.full(len(xs), 0.0 if greedy else 1.0, np.float32), cu=np.arange(len(xs) + 1, dtype=np.int32))
    n, nx = _run_verify(d)
    assert (n == 0).all() and nx.tolist() == xs


def test_verified_tokens_strides_and_streams():
    rng = np.random.default_rng(1)
    for pad in (1, 8):
        d = _logits(rng, [4, 2, 0, 7], 3000, "bf16", pad=pad)
        _check_verify(d)
    s = _torch().cuda.Stream()
    a, b = _run_verify(d), _run_verify(d, stream=s)
    assert np.array_equal(a, b)


def test_verified_tokens_degenerate_rows():
    torch = _torch()
    rng = np.random.default_rng(2)
    V = 5000
    d = _logits(rng, [3] * 12, V, "f32")
    p, q, cu, inf = d["p"], d["q"], d["cu"], float("inf")
    d["tau"][10] = 0.0
    d["tau"][11] = float("nan")
    q[0:3] = p[0:3]                                                  # 0: draft = target, everything accepted
    p[cu[1]] = -inf                                                  # 1: nothing possible: rejected (r Q > 0), next 0
    d["r"][3] = 0.5
    p[cu[2], :] = -inf; p[cu[2], 4321] = -3.4e38                     # 2: one finite logit, the type's lowest
    d["tok"][6], d["r"][6] = 17, 0.5
    p[cu[3], 100] = inf                                              # 3: an infinite logit takes all
    d["tok"][9], d["r"][9] = 5, 0.999
    q[9, 5] = 30.0
    p[cu[4], ::2] = float("nan")                                     # 4: NaN counts as -inf
    p[cu[5]:cu[6], 1000:] = -inf                                     # 5: a masked vocabulary
    d["tok"][18:21] = [-4, V + 9, 2]                                 # 6: tokens out of range are clamped
    p[cu[7]:cu[8]] = -3.4028234663852886e38                          # 7: every logit at the type's lowest value: uniform
    d["tau"][8], d["tau"][9] = 1e-3, 1e4
    p[cu[10]:cu[11], 77] = 50.0; p[cu[10]:cu[11], 4000] = 50.0       # 10: greedy, equal largest logits: the first
    d["tok"][30:33] = [77, 77, 4000]
    n, nx = _check_verify(d)
    assert n[0] == 3 and n[1] == 0 and nx[1] == 0 and nx[2] == 4321 and n[2] == 0 and nx[3] == 100 and n[3] == 0
    assert n[10] == 2 and nx[10] == 77 and 0 <= nx[7] < V


def test_verified_tokens_residual_that_vanishes():
    """Q >= P everywhere after rounding, yet rejected: the draw is from P."""
    V = 64
    d = _logits(np.random.default_rng(3), [1], V, "f32")
    d["p"][:] = 0.0
    d["q"][:] = 0.0
    d["r"][0] = 1.0                                                  # r Q <= P holds: accepted, drawn from row 1
    n, _ = _run_verify(d)
    assert n[0] == 1
    d["r"][0] = np.float32(1.5)                                      # (outside [0, 1): forces the rejection)
    n, nx = _run_verify(d)
    assert n[0] == 0 and nx[0] == int(np.argmin(d["noise"][0]))


def test_emitted_tokens_follow_the_target():
    """With k = 1 the first emitted token is distributed as softmax(p / tau), whatever the draft."""
    torch = _torch()
    rng = np.random.default_rng(4)
    V, N = 8, 4096
    lp, lq = 1.5 * rng.standard_normal(V), 1.5 * rng.standard_normal(V)
    want = np.exp(lp / 0.8) / np.exp(lp / 0.8).sum()
    qd = np.exp(lq / 0.8) / np.exp(lq / 0.8).sum()
    counts = np.zeros(V)
    for _ in range(12):
        tok = rng.choice(V, size=N, p=qd).astype(np.int32)
        d = dict(p=torch.tensor(np.broadcast_to(lp.astype(np.float32), (2 * N, V)).copy()), q=torch.tensor(np.broadcast_to(lq.astype(np.float32), (N, V)).copy()),
                 tok=tok, r=rng.random(N, dtype=np.float32), noise=rng.exponential(size=(N, V)).astype(np.float32), tau=np.full(N, 0.8, np.float32),
                 cu=np.arange(0, 2 * N + 1, 2).astype(np.int32))
        n, nx = _run_verify(d)
        counts += np.bincount(np.where(n == 1, tok, nx), minlength=V)
    got = counts / counts.sum()
    assert (np.abs(got - want) < 5 * np.sqrt(want * (1 - want) / counts.sum()) + 1e-4).all(), (got, want)


# ------------------------------------------------------------------------- graphs ----
def test_a_step_replays_from_a_graph():
    torch = _torch()
    b = _Batch([5, 5], [700, 300], 8, 2, 64, 16, "bf16", seed=21)
    q, k, v, table, cu, kv = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV), _i32(b.table), _i32(b.cu), _i32(b.kv)
    out, lse = torch.empty((10, 8, 64), dtype=q.dtype, device=DEV), torch.empty((10, 8), device=DEV)
    ws = torch.empty(B.sd_attend_workspace_bytes(q, k, table), dtype=torch.uint8, device=DEV)
    d = _logits(np.random.default_rng(8), [4, 4], 20000, "bf16")
    t = {n: torch.as_tensor(x).to(DEV) for n, x in d.items()}
    n, nx = (torch.empty(2, dtype=torch.int32, device=DEV) for _ in range(2))
    vws = torch.empty(B.sd_verify_logits_workspace_bytes(t["p"], t["q"], t["tau"]), dtype=torch.uint8, device=DEV)

    def step(stream):
        B.sd_attend(q, k, v, cu, kv, table, out, b.scale, lse=lse, ws=ws, stream=stream)
        B.sd_verify_logits(t["p"], t["q"], t["tok"], t["r"], t["noise"], t["tau"], t["cu"], n, nx, vws, stream=stream)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(s)
    for i in range(4):
        q.copy_(b.q.to(DEV) * (1 + 0.25 * i))
        t["r"].uniform_(0.0, 1.0)
        for x in (out, lse):
            x.fill_(-7.0)
        n.fill_(-7), nx.fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, n, nx)]
        step(None)
        torch.cuda.synchronize()
        for a, c in zip(got, (out, lse, n, nx)):
            assert torch.equal(a, c)
