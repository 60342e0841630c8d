"""Dense attention and the cache at the edges of what their documentation allows:
lengths past a block table, junk in masked places, rows of few keys anywhere in a
pack, exponents outside their range, NaN that is attended."""
import pytest
import torch

import dense_ref as R
from paper_2609_38978_amd import park as P
from test_gpu_cache import check_cached, filled, ints, same_pages, tables
from test_gpu_dense import rand, run

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("page,d", [(16, 64), (64, 128)])
@pytest.mark.parametrize("Nq", [1, 10, 150])
@pytest.mark.parametrize("kind", ["causal", "bias", "prefix", "all keys"])
def test_sequences_longer_than_their_table(kind, Nq, page, d):
    # queries stand at lens - q_lens + i whatever the table holds; tokens past it
    # are left out, and the status word says so
    gen = torch.Generator(device="cuda").manual_seed(51)
    B, Hq, Hkv, mp = 4, 4, 2, 5
    T = mp * page
    table, n = tables(gen, B, mp)
    cache = filled(gen, n, Hkv, page, d)
    # (the third is as long as its table, the last one's queries all stand past it)
    lens = [T + 7, T - 3, T, T + 2 * Nq + 40]
    ql = [max(1, Nq - 3), Nq, Nq, Nq]
    opts = {"bias": dict(slopes=torch.tensor([0.5, 0.1, 0.03, 0.0], device="cuda"), softcap=9.0),
            "prefix": dict(prefix=ints([T + 5, 3, T, 2 * T])), "all keys": dict(causal=False),
            "causal": {}}[kind]
    Q = rand(gen, B, Hq, Nq, d, BF)

    def attend(lens, ql):
        out, lse = torch.full((B, Hq, Nq, d), 9.0, device="cuda"), torch.full((B, Hq, Nq), 9.0, device="cuda")
        P.park_cache_attention(Q, cache, table, ints(lens), q_lens=ints(ql), out=out, lse=lse, **opts)
        check_cached(Q, cache, table, lens, ql, out, lse, **opts)

    attend(lens, ql)
    with pytest.raises(P.ParkError) as ei:
        P.park_check(cache["status"])
    assert ei.value.status == P.PARK_ERR_NUMERIC and "page" in str(ei.value)
    # no query reads past a table here: sequences end with it, or have no query
    attend([T, T - 3, T, T + 1], [Nq, Nq, 1, 0])
    P.park_check(cache["status"])


def test_the_longest_length():
    gen = torch.Generator(device="cuda").manual_seed(52)
    table, n = tables(gen, 1, 3)
    cache = filled(gen, n, 2, 32, 64)
    Q = rand(gen, 1, 2, 3, 64, BF)
    out, lse = torch.full((1, 2, 3, 64), 9.0, device="cuda"), torch.full((1, 2, 3), 9.0, device="cuda")
    P.park_cache_attention(Q, cache, table, ints([2 ** 31 - 1]), out=out, lse=lse)
    check_cached(Q, cache, table, [2 ** 31 - 1], [3], out, lse)


def relative_cap(Q, K, V, dO, opts, ok):
    """R.attention with the bounds of a cap whose tanh is off by 5 roundings (of
    scale / cap, of the product with it, of the sum x + x z p, of the product with
    the cap, and of the polynomial: 2^-21 together), relative, for scores far below
    the cap: those of no cap, and 2^-21 |x| more for each score."""
    val, tol = R.attention(Q, K, V, dO, **opts)
    plain = {k: v for k, v in opts.items() if k != "softcap"}
    tol = R.attention(Q, K, V, dO, **plain)[1]
    G = Q.shape[1] // K.shape[1]
    s = Q.shape[-1] ** -0.5 * (Q.double() @ K.double().repeat_interleave(G, 1).transpose(-1, -2))
    top = torch.where(ok[:, None], s.abs(), 0.0).amax(-1)
    more = 2 * 2.0 ** -21 * top  # of a probability, relative: its own and its normaliser's
    vabs = torch.where(ok.any(1)[:, None, :, None], V, 0.0).double().abs().repeat_interleave(G, 1)
    p = torch.exp(torch.where(ok[:, None], s, -INF) - val["lse"][..., None])
    p = torch.where(ok[:, None], p, 0.0) * 1.01
    tol["O"] = tol["O"] + 1.01 * more[..., None] * (p @ vabs)
    tol["lse"] = tol["lse"] + more
    return val, tol


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64)])
@pytest.mark.parametrize("where", ["masked keys", "padded queries"])
def test_large_scores_beside_small_ones_under_a_large_cap(where, dtype, d):
    # a key that nobody attends, or a query of no document, with scores about the
    # cap's size in every tile: the others keep a tanh of relative error
    gen = torch.Generator(device="cuda").manual_seed(53)
    B, H, N, cap = 2, 2, 300, 1e6
    Q, K, V = (rand(gen, B, H, N, d, dtype) for _ in range(3))
    kd = torch.zeros(B, N, dtype=torch.int32, device="cuda")
    qd = kd.clone()
    if where == "masked keys":
        kd[:, 5::16] = -1
        K[:, :, 5::16] *= 1e6
    else:
        qd[:, 5::16] = -1
        Q[:, :, 5::16] *= 1e6
    opts = dict(softcap=cap, q_doc=qd, k_doc=kd)
    ok = R.allowed(B, N, N, "cuda", q_doc=qd, k_doc=kd)
    val, tol = relative_cap(*(torch.where((i >= 0)[:, None, :, None], t, 0.0) for t, i in
                              ((Q, qd), (K, kd), (V, kd))), None, opts, ok)
    got = run(Q, K, V, None, opts)
    for n in got:
        R.check(n, got[n], val[n], tol[n])


@pytest.mark.parametrize("Nq", [1, 40])
def test_large_scores_behind_a_cached_sequence(Nq):
    # what stands behind the last token (an earlier sequence's, or nothing yet) has
    # scores about the cap's size
    gen = torch.Generator(device="cuda").manual_seed(54)
    table, n = tables(gen, 1, 3)
    cache = filled(gen, n, 2, 64, 64)
    T = 70
    last = int(table[0, 1])
    cache["k"][last, :, T - 64:] = 0x7e  # 448
    cache["k_exp"][last] = 0
    first = cache["k"][last, :, :T - 64].view(R.F8)
    first.copy_(torch.randn(2, T - 64, 64, generator=gen, device="cuda").to(R.F8))
    Q = rand(gen, 1, 4, Nq, 64, BF)
    Q[..., 0] = 500.0
    cache["k"][..., 0][cache["k"][..., 0] != 0x7e] = 0
    out, lse = torch.full((1, 4, Nq, 64), 9.0, device="cuda"), torch.full((1, 4, Nq), 9.0, device="cuda")
    cap = 3e4
    P.park_cache_attention(Q, cache, table, ints([T]), softcap=cap, out=out, lse=lse)
    k, v, there = R.cached_kv(cache, table, ints([T]))
    pos = torch.arange(Nq, device="cuda")[None] + T - Nq
    ok = there[:, None, :] & (torch.arange(k.shape[2], device="cuda") <= pos[..., None])
    k, v = (torch.where(there[:, None, :, None], t, 0.0) for t in (k, v))
    val, tol = relative_cap(Q, k, v, None, dict(softcap=cap, ok=ok, pos=pos), ok)
    u = R.attention(Q, k, v, ok=ok, pos=pos, u_out=2.0 ** -24)[1]
    bf = R.attention(Q, k, v, ok=ok, pos=pos)[1]
    R.check("O", out, val["O"], tol["O"] - bf["O"] + u["O"])
    R.check("lse", lse, val["lse"], tol["lse"])


JUNK = (3e4, -2e3, NAN, INF, -INF)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64), (F, 128)])
@pytest.mark.parametrize("cap", [0.0, 50.0, 1e6])
@pytest.mark.parametrize("kind", ["padded", "scattered", "few"])
def test_masked_places_change_no_bit(kind, cap, dtype, d):
    # whatever stands in tokens of no document, every other row has the same bits
    gen = torch.Generator(device="cuda").manual_seed(55)
    B, Hq, Hkv, Nq, Nk = (2, 4, 2, 5, 1500) if kind == "few" else (2, 4, 2, 420, 420)
    Q, dO = (rand(gen, B, Hq, Nq, d, dtype) * 2 for _ in range(2))
    K, V = (rand(gen, B, Hkv, Nk, d, dtype) * 2 for _ in range(2))
    qd, kd = (torch.zeros(B, n, dtype=torch.int32, device="cuda") for n in (Nq, Nk))
    if kind == "padded":
        qd[0, 300:], kd[0, 250:], qd[1, 77:], kd[1, 77:] = -1, -1, -1, -1
    else:
        qd[:, 3::7], kd[:, 5::11] = -1, -1
    opts = dict(softcap=cap, q_doc=qd, k_doc=kd)
    at = lambda i: (i < 0)[:, None, :, None]  # noqa: E731
    want = run(*(torch.where(at(i), torch.zeros((), dtype=dtype, device="cuda"), t)
                 for t, i in ((Q, qd), (K, kd), (V, kd), (dO, qd))), opts)
    for bad in JUNK:
        x = torch.tensor(bad, dtype=dtype, device="cuda")
        got = run(*(torch.where(at(i), x, t) for t, i in ((Q, qd), (K, kd), (V, kd), (dO, qd))), opts)
        for n in want:
            same = torch.equal(got[n], want[n])
            assert same, (n, bad)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F, 64), (F, 128)])
@pytest.mark.parametrize("Nq", [4, 300])
@pytest.mark.parametrize("cap", [0.0, 6.0])
def test_a_row_does_not_depend_on_other_queries(cap, Nq, dtype, d):
    # O, lse and dQ of a row have the same bits beside other queries
    gen = torch.Generator(device="cuda").manual_seed(56)
    Q, dO = (rand(gen, 1, 4, Nq, d, dtype) for _ in range(2))
    K, V = (rand(gen, 1, 2, 1100, d, dtype) for _ in range(2))
    opts = dict(softcap=cap, causal=True)
    want = run(Q, K, V, dO, opts)
    other = torch.arange(Nq, device="cuda") % 3 == 1
    for size in (0.0, 1.5, 60.0):
        q = torch.where(other[:, None], rand(gen, 1, 4, Nq, d, dtype, spread=size), Q)
        got = run(q, K, V, dO, opts)
        for n in ("O", "lse", "dQ"):
            same = torch.equal(got[n][:, :, ~other], want[n][:, :, ~other])
            assert same, (n, size)


@pytest.mark.parametrize("Nq", [1, 90])
@pytest.mark.parametrize("cap", [0.0, 50.0])
def test_the_rest_of_a_page_changes_no_bit(cap, Nq):
    gen = torch.Generator(device="cuda").manual_seed(57)
    B, Hq, Hkv, d, page, mp = 3, 4, 2, 64, 64, 20
    lens = [1203, 90, 1025]
    table, n = tables(gen, B, mp)
    cache = filled(gen, n, Hkv, page, d)
    Q = rand(gen, B, Hq, Nq, d, BF) * 2
    behind = torch.zeros(n, page, dtype=torch.bool, device="cuda")
    for b in range(B):
        for t in range(mp):
            behind[int(table[b, t]), max(0, min(page, lens[b] - t * page)):] = True
    outs = []
    for byte in (0, 0x7e, 0xfe, 0x7f):
        for side in ("k", "v"):
            cache[side][behind[:, None, :, None].expand_as(cache[side])] = byte
        outs.append(P.park_cache_attention(Q, cache, table, ints(lens), softcap=cap, want_lse=True))
    for O, lse in outs[1:]:
        same = torch.equal(O, outs[0][0]) and torch.equal(lse, outs[0][1])
        assert same


@pytest.mark.parametrize("e", [-128, -119, -111, -110, 119, 127])
@pytest.mark.parametrize("Nq", [2, 50])
def test_exponents_past_their_range(Nq, e):
    # a page's exponent is read as if within [-110, 119], of keys and of values
    gen = torch.Generator(device="cuda").manual_seed(58)
    d, page = 64, 16
    c = min(max(e, -110), 119)
    table = ints([[2, 0, 1]])
    Q = rand(gen, 1, 2, Nq, d, BF)
    pos = torch.arange(Nq, device="cuda")[None] + 41 - Nq
    cache = filled(gen, 3, 1, page, d)
    e0 = cache["v_exp"].clone()
    for side in ("v", "k"):
        cache["v_exp"].copy_(e0)
        cache["k_exp"].copy_(e0)
        cache[side + "_exp"].fill_(e)
        # values q 2^e with q below 2, so that 2^119 q is finite
        cache[side].copy_(torch.randint(0, 0x40, cache[side].shape, generator=gen, device="cuda"))
        k, v, there = R.cached_kv(cache, table, ints([41]))
        ok = there[:, None, :] & (torch.arange(48, device="cuda") <= pos[..., None])
        unit = cache[side][table.long()].view(R.F8).double().transpose(1, 2).reshape(1, 1, 48, d)
        out, lse = torch.empty(1, 2, Nq, d, device="cuda"), torch.empty(1, 2, Nq, device="cuda")
        q = Q if side == "v" else Q * 2.0 ** (-c if c < 0 else -100)  # (bf16: exact)
        scale = d ** -0.5 * (1.0 if side == "v" or c < 0 else 2.0 ** (100 - c))
        P.park_cache_attention(q, cache, table, ints([41]), out=out, lse=lse, scale=scale)
        # (relative to 2^c: the bounds have an absolute 1e-30)
        val, tol = R.attention(Q, k if side == "v" else unit, unit if side == "v" else v, ok=ok, pos=pos,
                               u_out=2.0 ** -24)
        R.check("lse", lse, val["lse"], tol["lse"])
        R.check("O", out.double() * (2.0 ** -c if side == "v" else 1.0), val["O"], tol["O"])


def few_keys(Q, K, V, dO, ok, cap):
    """dQ, dK and their bounds where D is formed from its definition: what is left is
    the rounding of dS and of the result (2^-8 each) and float sums (d + 16 roundings
    of 2^-24 of P (|dO||v| + sum P |dO||v|), and as much for P's own)."""
    B, Hq, Nq, d = Q.shape
    Hkv, Nk = K.shape[1:3]
    ok = ok[:, None]
    q, g = Q.double(), dO.double()
    k, v = (t.double().repeat_interleave(Hq // Hkv, 1) for t in (K, V))
    s = d ** -0.5 * (q @ k.transpose(-1, -2))
    t = torch.tanh(s / cap) if cap else torch.zeros_like(s)
    x = torch.where(ok, cap * t if cap else s, -INF)
    p = torch.where(ok, torch.exp(x - torch.logsumexp(x, -1, keepdim=True)), 0.0)
    dp, mag = g @ v.transpose(-1, -2), g.abs() @ v.abs().transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * (1 - t * t)
    # scores are off by d 2^-24 |q||k| scale (and 4e-7 of the cap): so is P, relative
    size = torch.where(ok, q.abs() @ k.abs().transpose(-1, -2), 0.0).amax(-1, keepdim=True)
    es = 2 * (d + 16) * 2.0 ** -24 * (1 + d ** -0.5 * size) + (8e-7 * cap if cap else 0.0)
    eds = 2.0 ** -8 * ds.abs() + (2 * es + (d + 16) * 2.0 ** -22) * p * (mag + (p * mag).sum(-1, keepdim=True))
    heads = lambda y: y.view(B, Hkv, Hq // Hkv, Nk, d).sum(2)  # noqa: E731
    dq, edq = d ** -0.5 * (ds @ k), d ** -0.5 * (eds @ k.abs())
    dk, edk = (d ** -0.5 * heads(y) for y in (ds.transpose(-1, -2) @ q, eds.transpose(-1, -2) @ q.abs()))
    return (dq, edq * 1.01 + 2.0 ** -8 * dq.abs() + 1e-30), (dk, edk * 1.01 + 2.0 ** -8 * dk.abs() + 1e-30)


def check_few(Q, K, V, dO, opts, rows=None, keys=None):
    B, Nq, Nk = Q.shape[0], Q.shape[2], K.shape[2]
    got = run(Q, K, V, dO, opts)
    ok = R.allowed(B, Nq, Nk, "cuda", **{k: v for k, v in opts.items() if k != "softcap"})
    (dq, eq), (dk, ek) = few_keys(Q, K, V, dO, ok, opts.get("softcap"))
    r = slice(None) if rows is None else rows
    c = slice(None) if keys is None else keys
    R.check("dQ", got["dQ"][:, :, r], dq[:, :, r], eq[:, :, r])
    R.check("dK", got["dK"][:, :, c], dk[:, :, c], ek[:, :, c])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1, 2, 3, 4, 7, 8])
def test_gradients_of_short_documents_anywhere(size, d):
    # documents of a few tokens at every place of a pack
    gen = torch.Generator(device="cuda").manual_seed(59)
    B, Hq, Hkv, N = 2, 6, 2, 333
    Q, dO = (rand(gen, B, Hq, N, d, BF) for _ in range(2))
    K, V = (rand(gen, B, Hkv, N, d, BF) for _ in range(2))
    ids = (torch.arange(N, device="cuda", dtype=torch.int32) // size).expand(B, N).contiguous()
    for more in (dict(causal=True), dict(softcap=20.0), dict(causal=True, prefix=ints([40, 333])), {}):
        check_few(Q, K, V, dO, dict(q_doc=ids, k_doc=ids, **more))


def test_gradients_of_documents_in_pieces():
    # a document of which a row sees a few keys around its own place and others far
    # away (in front of it, or behind): D is not that of the near ones alone
    gen = torch.Generator(device="cuda").manual_seed(65)
    Q, K, V, dO = (rand(gen, 1, 2, 400, 64, BF) for _ in range(4))
    ids = torch.arange(400, device="cuda", dtype=torch.int32) % 100 // 5
    for more in (dict(causal=True), {}):
        opts = dict(q_doc=ids[None].contiguous(), k_doc=ids[None].contiguous(), **more)
        got = run(Q, K, V, dO, opts)
        val, tol = R.attention(Q, K, V, dO, **opts)
        for n in got:
            R.check(n, got[n], val[n], tol[n])


@pytest.mark.parametrize("N", [700, 9000])
def test_gradients_of_short_documents_after_a_long_one(N):
    gen = torch.Generator(device="cuda").manual_seed(60)
    Hq, Hkv, d = (4, 2, 64) if N < 1000 else (1, 1, 64)
    Q, dO = (rand(gen, 1, Hq, N, d, BF) for _ in range(2))
    K, V = (rand(gen, 1, Hkv, N, d, BF) for _ in range(2))
    long = N - 101
    ids = torch.cat([torch.zeros(long, device="cuda"), 1 + torch.arange(101, device="cuda") // 4]).int()[None]
    short = torch.arange(long, N, device="cuda")
    for more in (dict(causal=True), {}):
        check_few(Q, K, V, dO, dict(q_doc=ids, k_doc=ids, **more), short, short)


def test_gradients_of_queries_with_few_keys_of_their_own():
    # keys and queries of different counts: eight keys of each query's document
    gen = torch.Generator(device="cuda").manual_seed(61)
    B, Hq, Hkv, Nq, Nk, d = 2, 3, 1, 150, 400, 128
    Q, dO = (rand(gen, B, Hq, Nq, d, BF) for _ in range(2))
    K, V = (rand(gen, B, Hkv, Nk, d, BF) for _ in range(2))
    kd = (torch.arange(Nk, device="cuda", dtype=torch.int32) // 8).expand(B, Nk).contiguous()
    qd = torch.randint(-1, 55, (B, Nq), generator=gen, device="cuda", dtype=torch.int32)
    check_few(Q, K, V, dO, dict(q_doc=qd, k_doc=kd))
    check_few(Q, K, V, dO, dict(q_doc=qd, k_doc=kd, causal=True))


@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("byte", [0x7f, 0xff])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("Nq", [1, 150])
def test_attended_nan_of_a_cache_is_seen(Nq, d, page, byte, side):
    # in a whole tile, in a partial one at the end, and where a causal limit falls;
    # the longest sequence is read in parts
    gen = torch.Generator(device="cuda").manual_seed(62)
    B, Hq, Hkv, lens = 3, 4, 2, [6001, 205, 400]
    table, n = tables(gen, B, -(-6001 // page) + 1)
    cache = filled(gen, n, Hkv, page, d)
    Q = rand(gen, B, Hq, Nq, d, BF)
    places = [(0, 0, 70, 3), (0, 1, 5998, d - 1), (1, 0, 204, 0), (1, 1, 130, 17), (2, 0, 0, 33)]
    for b, h, j, c in places:
        cache[side][int(table[b, j // page]), h, j % page, c] = byte
    O, lse = P.park_cache_attention(Q, cache, table, ints(lens), want_lse=True, out_dtype=F)
    want_o = torch.zeros(B, Hq, Nq, d, dtype=torch.bool, device="cuda")
    want_l = torch.zeros(B, Hq, Nq, dtype=torch.bool, device="cuda")
    for b, h, j, c in places:
        sees = torch.arange(Nq, device="cuda") + lens[b] - Nq >= j
        for hq in (2 * h, 2 * h + 1):
            want_o[b, hq] |= sees[:, None] & ((torch.arange(d, device="cuda") == c) if side == "v" else True)
            want_l[b, hq] |= sees & (side == "k")
    assert torch.equal(O.isnan(), want_o) and torch.equal(lse.isnan(), want_l)
    # and what is beside them is right
    k, v, there = R.cached_kv(cache, table, ints(lens))
    k, v = k.nan_to_num(0.0), v.nan_to_num(0.0)
    for b in range(B):
        pos = torch.arange(Nq, device="cuda")[None] + lens[b] - Nq
        ok = there[b][None, None] & (torch.arange(k.shape[2], device="cuda") <= pos[..., None])
        val, tol = R.attention(Q[b:b + 1], k[b:b + 1], v[b:b + 1], ok=ok, pos=pos, u_out=2.0 ** -24)
        f = ~want_o[b:b + 1]
        R.check("O", O[b:b + 1][f], val["O"][f], tol["O"][f])


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_a_nan_appended_is_attended(dtype):
    # from the input through the pages to the output
    gen = torch.Generator(device="cuda").manual_seed(63)
    table, n = tables(gen, 1, 4)
    cache = P.make_kv_cache(n, 1, 32, 64)
    K, V = (rand(gen, 1, 1, 100, 64, dtype) for _ in range(2))
    V[0, 0, 40, 7], V[0, 0, 90, 9] = INF, NAN
    P.park_cache_append(cache, K, V, table, ints([0]))
    O = P.park_cache_attention(rand(gen, 1, 1, 100, 64, BF), cache, table, ints([100]))[0, 0]
    assert O[40:, 7].isnan().all() and O[90:, 9].isnan().all()
    O[40:, 7], O[90:, 9] = 0.0, 0.0
    assert O.isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F], ids=["bf16", "f32"])
def test_append_at_the_end_of_the_range(dtype):
    # 448 2^119 is the largest value a page holds; what rounds to more becomes NaN,
    # as infinities do, and leaves its neighbours alone
    x = torch.zeros(1, 1, 2, 64)
    x[0, 0, 0, :11] = torch.tensor([448.0, 456.0, 464.0, 472.0, 480.0, 508.0, -464.0, -472.0, 440.0, 100.0, 2.0])
    x[0, 0, 1, :3] = torch.tensor([0.015625, 2.0 ** -9, 2.0 ** -10])  # normal, subnormal, half of that: to even
    x = (x.double() * 2.0 ** 119).to(dtype).cuda()
    assert x.isfinite().all()
    cache = P.make_kv_cache(1, 1, 16, 64)
    want = R.append(cache, x, -x, torch.tensor([[0]]), [0], [2])
    P.park_cache_append(cache, x, -x, ints([[0]]), ints([0]))
    same_pages(cache, want)
    nan = cache["k"][0, 0, 0, :11].view(R.F8).float().isnan().tolist()
    assert nan == [False] * 3 + [True] * 3 + [False, True] + [False] * 3


def test_gradients_inside_an_autograd_function():
    # outputs carry no history of their own; a Function that keeps what the gradient
    # takes gives autograd the same gradients as the call itself
    gen = torch.Generator(device="cuda").manual_seed(66)
    opts = dict(causal=True, softcap=20.0)

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            O, lse = P.park_attention(q, k, v, want_lse=True, **opts)
            ctx.save_for_backward(q, k, v, O, lse)
            return O, lse

        @staticmethod
        def backward(ctx, dO, dlse):
            return P.park_attention_backward(dO.contiguous(), *ctx.saved_tensors, dlse=dlse.contiguous(), **opts)

    Q, w = (rand(gen, 2, 4, 130, 64, BF) for _ in range(2))
    K, V = (rand(gen, 2, 2, 130, 64, BF) for _ in range(2))
    leaves = [t.clone().requires_grad_() for t in (Q, K, V)]
    assert not P.park_attention(*leaves, **opts).requires_grad
    O, lse = Attention.apply(*leaves)
    ((O * w).sum() + 2 * lse.sum()).backward()
    o, l = P.park_attention(Q, K, V, want_lse=True, **opts)  # noqa: E741
    want = P.park_attention_backward(w, Q, K, V, o, l, dlse=torch.full_like(l, 2.0), **opts)
    for t, g in zip(leaves, want):
        same = torch.equal(t.grad, g)
        assert same
