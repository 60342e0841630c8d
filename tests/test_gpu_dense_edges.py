"""Dense attention and the cache at the edges of what their documentation allows:
lengths past a block table, junk in masked places, rows of few keys anywhere in a
pack, exponents outside their range, NaN that is attended."""
import pytest
import torch

import dense_ref as R
from paper_2609_38978_amd import park as P
from test_gpu_cache import check_cached, filled, ints, tables
from test_gpu_dense import rand

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
