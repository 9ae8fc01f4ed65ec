"""Operators of a served verification step where they can go wrong: masks and temperatures of verification, requests that a step refuses,
streams, weights of very different sizes, and a whole step in a graph."""
import numpy as np
import pytest
import test_gpu_serve as G

from oracle import serve_oracle as SO
from paper_2603_12617_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _torch():
    import torch
    return torch


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mask", [-1e5, -1e9, -1e10, -1e12, -1e15, -1e20, -1e30])
@pytest.mark.parametrize("tau", [(0.6, 1.2), (0.05, 0.3)])
@pytest.mark.parametrize("draft", [True, False])
def test_masks_that_are_finite(dtype, mask, tau, draft):
    """All places of a row but a few hundred hold a mask: whole segments of nothing else."""
    rng = np.random.default_rng(int(-np.log10(-mask)) + 40)
    V = 3 * 8192 + 100
    d = G._logits(rng, [2] * 40, V, dtype, draft, tau=tau)
    keep = rng.permutation(4000)[:300]
    hide = np.ones(V, bool)
    hide[keep] = False
    d["p"][:, hide] = mask
    if draft:
        d["q"][:, hide] = mask
    # drafts are drawn from their rows (a token of probability 1e-50 would be 0 in 32 bits, and then nothing is rejected)
    rows = d["q"] if draft else d["p"][np.setdiff1d(np.arange(120), d["cu"][1:] - 1)]
    heat = np.repeat(d["tau"], 2)[:, None]
    d["tok"] = (rows.double().numpy() / heat + rng.gumbel(size=(80, V))).argmax(1).astype(np.int32)
    print("case", dtype, mask, tau, draft, flush=True)
    _, nx = G._check_verify(d)
    assert np.isin(nx, keep).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", [3000, 20000])
@pytest.mark.parametrize("tau", [1e-4, 1e-6, 1e-8, 1e-9, 1e-12, 1e-20, 1e-36])
def test_small_temperatures(dtype, V, tau):
    """Temperatures at which a row is as good as greedy, but for logits that are equal."""
    rng = np.random.default_rng(V)
    d = G._logits(rng, [3] * 30, V, dtype, tau=(tau, tau))
    d["p"] += 5.0
    d["tok"] = d["q"].float().argmax(1).numpy().astype(np.int32)
    print("case", dtype, V, tau, flush=True)
    n, _ = G._check_verify(d)
    assert n.max() > 0


@pytest.mark.parametrize("shift", [-1e7, -7.3e5, 7.2e5, 7.3e5, 3e6, 1e7])
def test_logits_far_from_zero(shift):
    """A row's probabilities do not depend on a number that is added to all of its logits (these sums are exact)."""
    rng = np.random.default_rng(3)
    d = G._logits(rng, [2] * 40, 10000, "f32")
    d["p"], d["q"] = d["p"].round() + shift, d["q"].round() + shift
    d["p"][:, 5000:] -= 8.0
    print("case", shift, flush=True)
    G._check_verify(d)


@pytest.mark.parametrize("V", [700, 5000, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_residual_of_equal_rows_is_nothing(V, dtype):
    """The draft's row is the target's, and yet its draft is rejected (by a number outside [0, 1)): the draw is from the target's row."""
    rng = np.random.default_rng(V)
    d = G._logits(rng, [1] * 25, V, dtype)
    d["q"] = d["p"][d["cu"][:-1]].clone()
    d["r"][:] = 3.0
    n, nx = G._check_verify(d)
    assert (n == 0).all() and len(set(nx.tolist())) > 5


@pytest.mark.parametrize("V", [64, 5000, 20000])
def test_residual_without_the_only_possible_token(V):
    """All of a row's mass lies on a draft without a distribution, which is rejected: it is drawn all the same."""
    rng = np.random.default_rng(V)
    d = G._logits(rng, [1] * 6, V, "f32", False)
    for b in range(6):
        at = int(rng.integers(0, V))
        row = d["cu"][b]
        d["p"][row] = -float("inf")
        d["p"][row, at] = 1.0
        d["tok"][b], d["r"][b] = at, 1.5
    n, nx = G._run_verify(d)
    assert (n == 0).all() and nx.tolist() == d["tok"].tolist()


@pytest.mark.parametrize("V", [40, 9000])
def test_infinite_logits_are_the_largest_number(V):
    """+inf counts as the largest float, so of the two the first place wins a greedy row."""
    big = np.finfo(np.float32).max
    p = np.random.default_rng(V).standard_normal((4, V)).astype(np.float32)
    p[0, [3, 10]] = big, np.inf
    p[1, [3, 10]] = np.inf, big
    p[2, [7, V - 1]] = big, np.inf
    p[3, [V - 2, V - 1]] = np.inf, np.inf
    none = np.zeros(0, np.int32)
    d = dict(p=_torch().tensor(p), q=None, tok=none, r=none.astype(np.float32), noise=np.ones((4, V), np.float32), tau=np.zeros(4, np.float32),
             cu=np.arange(5, dtype=np.int32))
    for tau in (0.0, 0.7):                                  # (equal noise: the first of equal weights)
        d["tau"][:] = tau
        assert G._run_verify(d)[1].tolist() == [3, 3, 7, V - 2], tau


@pytest.mark.parametrize("Bn,page", [(1, 16), (40, 16), (300, 7)])
def test_steps_of_which_nothing_stands(Bn, page):
    """accepted = -1: not even the token before the drafts is kept; below that it counts as -1."""
    rng = np.random.default_rng(Bn + page)
    st = G._pages_state(rng, Bn, page, 40, 3000, 150, rng.integers(0, 9, Bn), held_extra=2)
    acc = rng.integers(-1, 4, Bn)
    acc[0] = -1
    want = SO.pages(accepted=acc, page=page, **{**st, "nfree": int(st["nfree"][0])})
    assert want["length"][0] == st["length"][0]
    G._same_pages(G._run_pages(st, page, acc), want)
    G._same_pages(G._run_pages(st, page, np.where(acc == -1, -(1 << 31), acc)), want)


def test_a_refused_request_goes_on_where_it_stood():
    """Three requests, one page left for two that need one: the refused one keeps its length, and gets its tokens' slots a step later, once
    the third has given its page back."""
    page = 16
    st = dict(pages=np.array([1, 1, 1]), length=np.array([14, 14, 9]), add=np.array([5, 5, 5]), table=np.array([[4, -1], [2, -1], [1, -1]]),
              free=np.array([3, -1, -1, -1, -1]), nfree=np.array([1]))
    one = G._run_pages(st, page)
    assert one["kv"].tolist() == [19, 14, 14] and (one["slot"][5:10] == -1).all() and (one["slot"][10:] >= 0).all()
    refused = (one["kv"] == one["length"]) & (st["add"] > 0)
    assert refused.tolist() == [False, True, False]
    accepted = np.where(refused, -1, [1, 3, 0])              # (whatever verification says of rows that are not in the cache)
    add = np.array([0, 5, 0])
    length = one["length"].copy()
    length[2], accepted[2] = 0, -1                           # the third request has ended
    two = G._run_pages(dict(pages=one["pages"], length=length, add=add, table=one["table"], free=one["free"], nfree=one["nfree"]), page, accepted)
    assert two["length"].tolist() == [16, 14, 0] and two["kv"].tolist() == [16, 19, 0] and two["pages"].tolist() == [1, 2, 0]
    assert two["pos"].tolist() == [14, 15, 16, 17, 18] and two["slot"][:2].tolist() == [2 * page + 14, 2 * page + 15]
    assert two["slot"][2] == two["table"][1, 1] * page and (two["slot"] >= 0).all()


def test_a_long_chunk_among_many_requests():
    """One request of 4096 brings 600000 tokens: more than 2^31 / 4096, and no more than a step may have."""
    rng = np.random.default_rng(11)
    st = G._pages_state(rng, 4096, 16, 9, 9000, 100, rng.integers(0, 3, 4096))
    st["add"][7] = 600000                                    # (too long for its table: refused, and still its tokens have their places)
    want = SO.pages(page=16, **{**st, "nfree": 9000})
    assert want["cu"][8] - want["cu"][7] == 600000
    G._same_pages(G._run_pages(st, 16), want)


def test_new_tokens_beyond_32_bits_stay_in_the_arrays():
    """Sums of new tokens past 2^31 - 1 end there."""
    st = dict(pages=np.array([1, 1, 1, 0]), length=np.array([3, 3, 3, 0]), add=np.array([5, 0x7fffffff, 0x7ffffff0, 9]), table=np.array([[4, -1], [2, -1], [1, -1], [-1, -1]]),
              free=np.array([3, 0, -1, -1, -1]), nfree=np.array([2]))
    got = G._run_pages(st, 16, tokens=20)
    assert got["cu"].tolist() == [0, 5, 0x7fffffff, 0x7fffffff, 0x7fffffff] and got["kv"].tolist() == [8, 3, 3, 9] and got["nfree"].tolist() == [1]
    assert got["pos"].tolist() == [3, 4, 5, 6, 7] + [-1] * 15 and got["slot"][:5].tolist() == [67, 68, 69, 70, 71] and (got["slot"][5:] == -1).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("Bn,rows,heads,D", [(64, 1, 8, 80), (4, 130, 64, 64)])
def test_attention_small_weights_beside_a_large_one(dtype, Bn, rows, heads, D):
    """One key far above 131072 equal ones, each of them less than 2^-25 of it and 0.4 % together; all values are 1.  Whole requests of one
    token and chunks, both so many that keys are not split (which would bring the others to parts of their own)."""
    torch = _torch()
    n, page = 262144, 64
    k = torch.zeros((n // page, page, heads, D), dtype=G._dt(dtype), device=DEV)
    v = torch.ones_like(k)
    tail = (torch.arange(page, device=DEV) & 4) != 0
    k[:, ~tail, :, 0] = -1000.0                             # (weight 0: half of the keys, so that the small weights' sum, in float32, is not theirs)
    k[0, 0, :, 0] = 17.34375
    gap = float(k[0, 0, 0, 0])
    q = torch.zeros((Bn * rows, heads, D), dtype=k.dtype, device=DEV)
    q[:, :, 0] = 8.0
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).expand(Bn, -1).contiguous()     # (all requests on the same pages)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    ws = torch.empty(B.sd_attend_workspace_bytes(q, k, table), dtype=torch.uint8, device=DEV)
    print("case", dtype, Bn, rows, heads, D, flush=True)
    B.sd_attend(q, k, v, G._i32(np.arange(Bn + 1) * rows), G._i32([n] * Bn), table, out, 0.125, lse=lse, ws=ws)
    torch.cuda.synchronize()
    # Weights and the result are rounded once each, relative; weights below float16's normal numbers to 2^-25 of a scale on which the largest is
    # at least 2^7; values are added up 16 keys at a time, each sum of about 1 rounded or cut to 24 bits.
    tol = 2.1 * G.UNIT[dtype] + n * 2.0 ** -32 + n / 16 * 2.0 ** -23
    assert float((out.double() - 1.0).abs().max()) <= tol
    pos = n - rows + np.arange(rows)
    seen = (pos + 1) // 8 * 4 + np.maximum((pos + 1) % 8 - 4, 0)
    want = gap + np.log1p(seen * np.exp(-gap))
    assert np.abs(lse.double().cpu().numpy().reshape(Bn, rows, heads) - want[None, :, None]).max() <= gap * 2.0 ** -22 + 1e-5


def test_calls_follow_the_torch_operations_before_them():
    """Inside a stream's block the operators wait for what torch computes there, and torch for them."""
    torch = _torch()
    b = G._Batch([5, 33, 1], [900, 400, 2000], 8, 2, 128, 16, "bf16", seed=12)
    want, _ = b.gpu()
    q, k, v, table, cu, kv = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV), G._i32(b.table), G._i32(b.cu), G._i32(b.kv)
    ws = torch.empty(B.sd_attend_workspace_bytes(q, k, table), dtype=torch.uint8, device=DEV)
    late, out, copy = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    busy = torch.randn((4096, 4096), device=DEV)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            busy = torch.tanh(busy @ busy)                  # (some milliseconds)
        late.copy_(q)
        B.sd_attend(late, k, v, cu, kv, table, out, b.scale, ws=ws)
        copy.copy_(out)
    torch.cuda.synchronize()
    assert torch.equal(copy, want)


def test_a_whole_step_replays_from_a_graph():
    """Tables, cache writes, attention and verification, captured on torch's current stream."""
    torch = _torch()
    Bn, page, Hq, Hkv, D, k, V = 3, 16, 8, 2, 64, 4, 20000
    rng = np.random.default_rng(5)
    g = torch.Generator(device=DEV).manual_seed(5)
    st = G._pages_state(rng, Bn, page, 40, 30, 500, 5, held_extra=1)
    i = {n: G._i32(x) for n, x in st.items()}
    T, pool = Bn * (k + 1), len(st["free"])
    new = lambda *s: torch.full(s, -7, dtype=torch.int32, device=DEV)  # noqa: E731
    o = dict(pages=new(Bn), length=new(Bn), kv=new(Bn), nfree=new(1), cu=new(Bn + 1), slot=new(T), pos=new(T), n=new(Bn), next=new(Bn),
             table=i["table"], free=i["free"])
    bf = lambda *s: torch.randn(s, generator=g, device=DEV).to(torch.bfloat16)  # noqa: E731
    o["k"], o["v"], q = bf(pool, page, Hkv, D), bf(pool, page, Hkv, D), bf(T, Hq, D)
    o["out"], o["lse"], acc, kn, vn = torch.empty_like(q), torch.empty((T, Hq), device=DEV), new(Bn), bf(T, Hkv, D), bf(T, Hkv, D)
    d = {n: x if x is None else torch.as_tensor(x).to(DEV) for n, x in G._logits(rng, [k] * Bn, V, "bf16").items()}
    ws = torch.empty(B.sd_attend_workspace_bytes(q, o["k"], i["table"]), dtype=torch.uint8, device=DEV)
    vws = torch.empty(B.sd_verify_logits_workspace_bytes(d["p"], d["q"], d["tau"]), dtype=torch.uint8, device=DEV)

    def step():
        B.sd_pages(i["pages"], i["length"], i["add"], i["table"], i["free"], i["nfree"], page, o["pages"], o["length"], o["kv"], o["nfree"], o["cu"],
                   o["slot"], o["pos"], accepted=acc)
        B.sd_cache_store(kn, vn, o["slot"], o["k"], o["v"])
        B.sd_attend(q, o["k"], o["v"], o["cu"], o["kv"], i["table"], o["out"], D ** -0.5, lse=o["lse"], ws=ws)
        B.sd_verify_logits(d["p"], d["q"], d["tok"], d["r"], d["noise"], d["tau"], o["cu"], o["n"], o["next"], vws)

    acc.fill_(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(5):
        acc.copy_(G._i32(rng.integers(-1, k + 1, Bn)))
        for x in (q, kn, vn):
            x.copy_(bf(*x.shape))
        d["r"].uniform_(0.0, 1.0)
        before = {n: o[n].clone() for n in ("k", "v", "table", "free")}
        for n in ("pages", "length", "kv", "nfree", "cu", "slot", "pos", "n", "next", "out", "lse"):
            o[n].fill_(-7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {n: x.clone() for n, x in o.items()}
        for n, x in before.items():
            o[n].copy_(x)
        step()
        torch.cuda.synchronize()
        for n, x in o.items():
            assert torch.equal(got[n], x), (turn, n)
        want = SO.pages(accepted=acc.tolist(), page=page, **{**st, "nfree": 30})
        for n in ("pages", "length", "kv", "cu", "slot", "pos", "nfree"):
            assert got[n].tolist() == want[n].tolist(), (turn, n)
        assert all(got["table"][b, :m].tolist() == want["table"][b, :m].tolist() for b, m in enumerate(want["pages"]))
        assert (got["out"] != -7).all() and (got["n"] >= 0).all() and (got["next"] >= 0).all()


@pytest.mark.parametrize("Bn,width", [(1, 8), (1, 40), (1, 600), (2, 600), (70, 600)])
def test_attention_of_requests_without_rows(Bn, width):
    """An idle step: no request has a token, the batch is padded.  Nothing is written."""
    torch = _torch()
    q = torch.ones((5, 8, 64), dtype=torch.bfloat16, device=DEV)
    k = torch.ones((20, 16, 2, 64), dtype=torch.bfloat16, device=DEV)
    out, lse = torch.full_like(q, -7.0), torch.full((5, 8), -7.0, device=DEV)
    table = torch.zeros((Bn, width), dtype=torch.int32, device=DEV)
    ws = torch.full((B.sd_attend_workspace_bytes(q, k, table),), 0x01, dtype=torch.uint8, device=DEV)
    print("case", Bn, width, flush=True)
    for kv in (0, 16 * width):
        B.sd_attend(q, k, k, G._i32([0] * (Bn + 1)), G._i32([kv] * Bn), table, out, 0.125, lse=lse, ws=ws)
        torch.cuda.synchronize()
        assert (out == -7).all() and (lse == -7).all()


@pytest.mark.parametrize("new,kv", [([3], [40]), ([150], [400]), ([2], [3000])])
@pytest.mark.parametrize("scale", [1e-30, 1e-38, 1e-42, 1e-300])
def test_attention_scales_next_to_nothing(new, kv, scale):
    """Scores that are 0 after scaling: the mean of the keys that a row sees."""
    b = G._Batch(new, kv, 4, 2, 64, 16, "bf16", seed=2)
    b.scale = scale
    print("case", new, kv, scale, flush=True)
    b.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k,V", [([0], 7), ([1], 1), ([0, 3, 1, 8, 0], 4099), ([3] * 5, 8193), ([5, 70], 300), ([2, 2], 50257)])
@pytest.mark.parametrize("draft", [True, False])
def test_small_batches_leave_little_undecided(dtype, k, V, draft):
    """Over many batches of few requests, nine in ten are compared: rounding could have decided otherwise only in the others."""
    sure = all_of_them = 0
    for seed in range(max(4, 40 // len(k)) if V < 10000 else 8):
        d = G._logits(np.random.default_rng(1000 * seed + V), k, V, dtype, draft)
        n, nx = G._run_verify(d)
        host = lambda x: None if x is None else x.double().numpy()  # noqa: E731
        wn, wx, close = SO.verify_logits(host(d["p"]), host(d["q"]), d["tok"], d["r"], d["noise"], d["tau"], d["cu"])
        ok = close > 4e-5
        assert np.array_equal(n[ok], wn[ok]) and np.array_equal(nx[ok], wx[ok]), (seed, n, wn, nx, wx, close)
        sure += int(ok.sum())
        all_of_them += len(k)
    print("case", dtype, k, V, draft, "%d of %d" % (sure, all_of_them), flush=True)
    assert sure > 0.9 * all_of_them


@pytest.mark.parametrize("new,kv,D", [([1] * 64, list(range(200, 840, 10)), 128), ([5, 1], [300, 20], 256), ([150, 1], [400, 30], 256)])
def test_attention_with_more_than_64k_of_shared_memory_replays_from_a_graph(new, kv, D):
    """What such a launch asks the runtime for may be asked while a stream is captured."""
    torch = _torch()
    b = G._Batch(new, kv, 8, 8, D, 16, "bf16", seed=D)
    want, want_lse = b.gpu()
    q, k, v, table, cu, lengths = b.q.to(DEV), b.k.to(DEV), b.v.to(DEV), G._i32(b.table), G._i32(b.cu), G._i32(b.kv)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    ws = torch.empty(B.sd_attend_workspace_bytes(q, k, table), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    print("case", len(new), D, flush=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sd_attend(q, k, v, cu, lengths, table, out, b.scale, lse=lse, ws=ws)
    for _ in range(3):
        out.fill_(-7.0), lse.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
