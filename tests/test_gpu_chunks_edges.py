"""GPU tests of the caller's paged cache where its inputs leave the ordinary: bad pages that only some rows see, scores near
the ends of their format, calls on other streams, caches so long that a lost tile of keys is small beside the roundings."""
import numpy as np
import pytest
import torch

from oracle import chunks as K
from test_gpu_chunks import HALF_STEP, TINY, E, _batch, _check_attention, _dev, _f64, _tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2602_02192_b200 import binding
    return binding


def _positions(starts, lens, rows):
    """Position of every row; -1 for rows of no sequence."""
    t = np.full(rows, -1)
    for _, row, at in K.positions(starts, lens):
        t[row] = at
    return t


# ---- bad pages ------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,seqs,s,bad", [
    ((4, 1, 64), [(3, 40), (16, 24)], 1, [1]),               # 64 rows to a tile
    ((8, 2, 128), [(1, 9), (30, 30), (2, 50)], 1, [1]),      # one tile of 128 rows
    ((8, 2, 128), [(64, 64), (5, 70)], 0, [2]),              # two
    ((8, 2, 64), [(200, 300), (1, 1)], 0, [14, 9]),          # several items, every other one from its last keys to its first
    ((32, 8, 128), [(10, 9000)], 0, [562]),                  # long caches, cut among the CTAs
    ((32, 8, 128), [(20, 9000), (1, 700)], 0, [562]),
    ((32, 8, 128), [(40, 9000)], 0, [562, 561]),
    ((32, 8, 128), [(40, 9000)], 0, [3]),                    # a page that every row needs
    ((8, 2, 128), [(100, 40)], 0, [1]),                      # rows that see nothing
])
def test_a_bad_page_spoils_the_rows_that_need_it(B, heads, seqs, s, bad):
    Hq, Hkv, hd = heads
    starts, lens, table, n_pages = _tables(seqs, seed=21)
    n = int(starts[-1])
    rng = np.random.default_rng(22)
    pool = _dev(rng.normal(size=(n_pages, Hkv, 2, 16, hd))).bfloat16()
    q = _dev(rng.normal(size=(n, Hq, hd))).bfloat16()
    want, spread, scores = K.attend(_f64(pool), _f64(q), starts, lens, table, np.zeros(q.shape))
    t = _positions(starts, lens, n)
    needs = np.zeros(n, dtype=bool)
    needs[starts[s]:starts[s + 1]] = t[starts[s]:starts[s + 1]] >= 16 * min(bad)
    assert needs.any()
    for page in (-1, n_pages):
        spoiled = table.copy()
        spoiled[s, bad] = page
        chunks = _batch(B, starts, lens, spoiled, n, max(c for c, _ in seqs))
        got = _f64(B.echo_chunk_attention(chunks, q, pool))
        with pytest.raises(B.EchoError, match="a page id"):
            chunks.check()
        assert np.isnan(got[needs]).all()
        keep = ~needs
        _check_attention(got[keep], want[keep], spread[keep], scores[keep], np.maximum(t[keep] + 1, 0), 8.0, torch.bfloat16, hd)


# ---- status ---------------------------------------------------------------------------------------
def test_check_waits_for_calls_on_other_streams(B):
    pool = torch.zeros((2, 1, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.ones((1, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    one, start = np.array([1], np.int32), np.array([0, 1], np.int32)
    chunks = _batch(B, start, one, np.array([[9]], np.int32), 1, 1)
    side = torch.cuda.Stream()
    for sleep in (0, 200_000_000):                           # (the first time the kernels are loaded); a tenth of a second
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(sleep)
            B.echo_append_kv(chunks, None, k, v, pool)
        with pytest.raises(B.EchoError, match="a page id"):
            chunks.check()
        chunks.check()


def test_a_batch_that_says_no_new_tokens(B):
    """max_chunk = 0 with rows that no sequence has: nothing to do, and no error, nor a finding."""
    i32 = dict(dtype=torch.int32, device="cuda")
    chunks = B.KVChunks(torch.zeros(4, **i32), torch.full((3,), 5, **i32), torch.zeros((3, 1), **i32), 7, 0)
    pool = torch.ones((2, 2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = (torch.ones((7, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    out = torch.full_like(q, 7.0)
    assert B.echo_append_kv(chunks, q, k, v, pool, out=out) is out and bool((out == 7).all())
    assert B.echo_chunk_attention(chunks, q, pool, out=out) is out and bool((out == 7).all())
    chunks.check()
    assert bool((pool == 1).all())


# ---- scores near the ends of their format ---------------------------------------------------------
@pytest.mark.parametrize("heads,seqs", [
    ((4, 2, 64), [(5, 300), (9, 9)]),                        # 64 rows to a tile
    ((8, 2, 128), [(30, 1000), (1, 70)]),
    ((8, 2, 128), [(150, 700)]),
    ((8, 2, 64), [(130, 130), (40, 9000)]),
])
@pytest.mark.parametrize("dtype,size", [(torch.float16, 60000.0), (torch.float16, 20000.0), (torch.bfloat16, 1.5e19), (torch.bfloat16, 1e13),
                                        (torch.bfloat16, 5e4)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_near_the_ends_of_their_format(B, heads, seqs, dtype, size, sign):
    """One element of q and k makes the score, so that it is a product that fp32 holds to a rounding; neighbouring keys'
    scores lie so far apart that a row's largest has all of the probability: its value comes out as it is.  Every third row
    has ordinary queries beside them, whose scores are 0 here: it has the mean of the values."""
    Hq, Hkv, hd = heads
    starts, lens, table, n_pages = _tables(seqs, seed=23)
    n = int(starts[-1])
    rng = np.random.default_rng(24)
    pool = np.zeros((n_pages, Hkv, 2, 16, hd))
    pool[:, :, 1] = rng.normal(size=pool[:, :, 1].shape)
    # 64 sizes, a 128th of the largest apart; each position's at random
    pool[:, :, 0, :, 3] = sign * size * (1 - rng.integers(0, 64, size=pool[:, :, 0, :, 3].shape) / 128)
    pool = _dev(pool).to(dtype)
    q = torch.zeros((n, Hq, hd), dtype=dtype, device="cuda")
    q[..., 3] = size
    flat = np.arange(n) % 3 == 2
    q[torch.from_numpy(flat).cuda()] = 0
    chunks = _batch(B, starts, lens, table, n, max(c for c, _ in seqs))
    got = _f64(B.echo_chunk_attention(chunks, q, pool))
    chunks.check()
    want, spread, scores = K.attend(_f64(pool), _f64(q), starts, lens, table, np.zeros(q.shape))
    t = _positions(starts, lens, n)
    assert np.isfinite(want).all()
    # equal probabilities (of equal scores) are equal numbers of the format, at most 2^-8 apart from their fp32 values
    h = HALF_STEP[dtype]
    tol = h * np.abs(want) + spread * (1 + h) * (h + 2 * E * (t[:, None, None] + 17)) + 2 * TINY[dtype]
    assert np.all(np.abs(got - want) <= tol), np.argwhere(~(np.abs(got - want) <= tol))[:5]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_of_a_tile_that_hold_nothing_have_no_part_in_the_others(B, dtype):
    """100 query heads to a kv head leave 28 rows of each tile as an earlier call left them: with queries of any size in
    them, the results are the same bit for bit."""
    S, kv, hd, n = 200, 300, 128, 3
    starts, lens = np.arange(S + 1, dtype=np.int32) * n, np.full(S, kv, np.int32)
    pages = -(-kv // 16)
    rng = np.random.default_rng(37)
    table = rng.permutation(S * pages).reshape(S, pages).astype(np.int32)
    pool = _dev(rng.normal(size=(S * pages, 1, 2, 16, hd)) * 20).to(dtype)
    q = _dev(rng.normal(size=(S * n, 100, hd)) / 20).to(dtype)
    chunks = _batch(B, starts, lens, table, S * n, n)
    got = []
    for size in (0.0, 1e3, 6e4, float("inf")):               # scores of 0, 10^5, 10^7 and infinities
        B.echo_chunk_attention(chunks, torch.full((S * n, 128, hd), size, dtype=dtype, device="cuda"), pool)
        got.append(B.echo_chunk_attention(chunks, q, pool))
    chunks.check()
    assert all(torch.equal(got[0], x) for x in got[1:])


# ---- every tile of keys, once ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,seqs,q_size", [
    ((2, 1, 64), [(1, 33333)], 1.0),
    ((8, 8, 64), [(1, 30000)] * 3 + [(140, 4000)], 0.1),
    ((8, 8, 128), [(1, 20000)] * 4 + [(2, 17)], 1.0),
    ((8, 2, 64), [(20, 33000)], 0.1),                        # 80 rows
    ((8, 2, 128), [(70, 12000), (100, 5000)], 0.1),          # two tiles of rows, every other pair from the last keys to the first
    ((4, 4, 64), [(260, 9000)], 1.0),
])
def test_no_tile_of_a_long_cache_is_lost_or_taken_twice(B, heads, seqs, q_size, dtype):
    """The values of the 128 keys of a tile are 1 in one column, another for each tile (hd tiles long), and 0 elsewhere: a
    column of the result is the probability of its few tiles, and all roundings are relative to that.  What one tile adds is
    well above them, which is asserted."""
    Hq, Hkv, hd = heads
    starts, lens, table, n_pages = _tables(seqs, seed=25)
    n = int(starts[-1])
    rng = np.random.default_rng(26)
    pool = torch.zeros((n_pages, Hkv, 2, 16, hd), dtype=dtype, device="cuda")
    pool[:, :, 0] = _dev(rng.normal(size=(n_pages, Hkv, 16, hd))).to(dtype)
    for s, (_, kv) in enumerate(seqs):
        for p in range(-(-kv // 16)):
            pool[int(table[s, p]), :, 1, :, (p // 8) % hd] = 1
    q = _dev(rng.normal(size=(n, Hq, hd)) * q_size).to(dtype)
    chunks = _batch(B, starts, lens, table, n, max(c for c, _ in seqs))
    got = _f64(B.echo_chunk_attention(chunks, q, pool))
    chunks.check()
    h, row = HALF_STEP[dtype], 0
    k64, q64 = pool[:, :, 0].double(), q.double()
    for s, (c, kv) in enumerate(seqs):
        k = k64[torch.from_numpy(table[s, :-(-kv // 16)]).long().cuda()].transpose(0, 1).reshape(Hkv, -1, hd)[:, :kv]
        rows = q64[row:row + c].view(c, Hkv, -1, hd)
        seen = torch.arange(kv, device="cuda")[None] <= torch.arange(kv - c, kv, device="cuda")[:, None]
        z = torch.einsum("nhgd,hkd->nhgk", rows, k) / hd ** 0.5
        size = torch.einsum("nhgd,hkd->nhgk", rows.abs(), k.abs()) / hd ** 0.5
        p = torch.softmax(z.masked_fill(~seen[:, None, None], -np.inf), dim=-1)
        pad = -kv % 128
        tiles = torch.nn.functional.pad(p, (0, pad)).view(c, Hkv, -1, (kv + pad) // 128, 128).sum(dim=-1)
        want = torch.zeros((c, Hkv, Hq // Hkv, hd), dtype=torch.float64, device="cuda")
        want.index_add_(3, torch.arange(tiles.shape[3], device="cuda") % hd, tiles)
        d = 2 * E * (hd + 8) * size.amax(dim=-1, keepdim=True)
        tol = h * want + (1 + h) * want * (h + 2 * d + 2 * E * (kv + 16)) + TINY[dtype]
        if dtype == torch.float16:
            tol += p.amax(dim=-1, keepdim=True) * kv * 2.0 ** -31
        err = (torch.from_numpy(got[row:row + c]).cuda().view(want.shape) - want).abs()
        assert bool((err <= tol).all()), (s, (~(err <= tol)).nonzero()[:5])
        whole = tiles[..., :max((kv - c + 1) // 128, 0)]             # tiles that all rows see
        bound = tol.gather(3, (torch.arange(whole.shape[3], device="cuda") % hd).expand(whole.shape))
        assert whole.shape[3] == 0 or bool((whole > 2 * bound).double().mean() > 0.999)
        row += c


@pytest.mark.parametrize("heads,seqs", [
    ((4, 2, 64), [(1, 1), (5, 700), (12, 129)]),
    ((32, 8, 128), [(1, 9000), (16, 300)]),
    ((10, 2, 64), [(40, 2000), (130, 130), (1, 1001)]),
    ((64, 8, 128), [(70, 1500), (3, 129)]),
])
@pytest.mark.parametrize("size", [0.01, 1.0, 5.0])
def test_small_probabilities_in_half_precision(B, heads, seqs, size):
    """A probability is rounded by half of the format's step, or where it is below the normal numbers by 2^-25 of a scale on
    which the row's largest is at least 2^6: 2^-31 of that.  The other roundings are relative, as in the tests of the chunks."""
    Hq, Hkv, hd = heads
    starts, lens, table, n_pages = _tables(seqs, seed=35)
    n = int(starts[-1])
    rng = np.random.default_rng(36)
    pool = _dev(rng.normal(size=(n_pages, Hkv, 2, 16, hd))).half()
    q = _dev(rng.normal(size=(n, Hq, hd)) * size).half()
    chunks = _batch(B, starts, lens, table, n, max(c for c, _ in seqs))
    got = _f64(B.echo_chunk_attention(chunks, q, pool))
    chunks.check()
    want, spread, scores = K.attend(_f64(pool), _f64(q), starts, lens, table, np.zeros(q.shape))
    keys = _positions(starts, lens, n)[:, None, None] + 1
    h, top = HALF_STEP[torch.float16], float(pool.abs().max())
    d = 2 * E * (hd + 8) * scores[:, :, None]
    tol = h * np.abs(want) + (1 + h) * spread * (h + 2 * d + 2 * E * (keys + 16)) + TINY[torch.float16] + keys * 2.0 ** -31 * top
    assert np.all(np.abs(got - want) <= tol), np.argwhere(~(np.abs(got - want) <= tol))[:5]



# ---- workspaces -----------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,longest", [
    ((32, 8, 128), 1), ((32, 8, 128), 16), ((32, 8, 128), 17), ((32, 8, 128), 32), ((32, 8, 128), 33),       # 64 rows, 128, two tiles
    ((10, 2, 64), 1), ((10, 2, 64), 12), ((10, 2, 64), 13), ((10, 2, 64), 25), ((10, 2, 64), 26),
    ((128, 1, 64), 1), ((128, 1, 64), 2), ((48, 1, 128), 2), ((48, 1, 128), 3), ((7, 1, 128), 9),
])
def test_a_workspace_of_the_stated_size_is_enough(B, heads, longest):
    Hq, Hkv, hd = heads
    seqs = [(longest, 9000), (1, 1), (longest, longest + 2000), (longest, longest)]
    starts, lens, table, n_pages = _tables(seqs, seed=27)
    n = int(starts[-1])
    g = torch.Generator(device="cuda").manual_seed(28)
    pool = torch.randn((n_pages, Hkv, 2, 16, hd), generator=g, device="cuda").bfloat16()
    q = torch.randn((n, Hq, hd), generator=g, device="cuda").bfloat16()
    chunks = _batch(B, starts, lens, table, n, longest)
    want = B.echo_chunk_attention(chunks, q, pool)
    need = B.lib.echo_chunk_attention_workspace_bytes(longest, Hq, Hkv, hd)
    assert need % 4 == 0
    guard = 4096
    whole = torch.full((need + 2 * guard,), 0xA5, dtype=torch.uint8, device="cuda")
    got = B.echo_chunk_attention(chunks, q, pool, workspace=whole[guard:guard + need])
    chunks.check()
    assert torch.equal(got, want)
    assert bool((whole[:guard] == 0xA5).all()) and bool((whole[guard + need:] == 0xA5).all())
    assert bool((whole[guard:guard + need] != 0xA5).any())               # it was used
    with pytest.raises(B.EchoError, match="ECHO_ERR_INVALID"):
        B.echo_chunk_attention(chunks, q, pool, workspace=whole[guard:guard + need - 1], out=torch.empty_like(q))


def test_rows_in_front_of_the_first_sequence(B):
    """row_starts may begin behind row 0: the rows before are left as they are."""
    Hq, Hkv, hd, front = 8, 2, 64, 5
    starts, lens, table, n_pages = _tables([(3, 40), (0, 9), (70, 90)], seed=29)
    n = int(starts[-1])
    g = torch.Generator(device="cuda").manual_seed(30)
    pool = torch.randn((n_pages, Hkv, 2, 16, hd), generator=g, device="cuda").bfloat16()
    q, k, v = (torch.randn((n + front, H, hd), generator=g, device="cuda").bfloat16() for H in (Hq, Hkv, Hkv))
    pools = [pool.clone(), pool.clone()]
    plain, moved = _batch(B, starts, lens, table, n, 70), _batch(B, starts + front, lens, table, n + front, 70)
    a = B.echo_append_kv(plain, q[front:], k[front:], v[front:], pools[0])
    b = B.echo_append_kv(moved, q, k, v, pools[1], out=torch.full_like(q, 7.0))
    assert torch.equal(pools[0], pools[1]) and torch.equal(a, b[front:]) and bool((b[:front] == 7).all())
    x = B.echo_chunk_attention(plain, a, pools[0])
    y = B.echo_chunk_attention(moved, b, pools[0], out=torch.full_like(q, 7.0))
    assert torch.equal(x, y[front:]) and bool((y[:front] == 7).all())
    plain.check()
    moved.check()


# ---- waits ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("heads,seqs", [
    ((32, 8, 128), [(16, 300)] * 40),                        # 64 rows to a tile
    ((32, 8, 128), [(30, 500)] * 40),                        # one tile of 128 rows
    ((32, 8, 128), [(64, 900), (130, 5000)] * 8),            # two
    ((8, 8, 64), [(128, 400), (3, 9000)] * 12),
])
def test_a_wait_that_runs_out_is_reported_and_leaves_the_device_as_it_was(B, heads, seqs):
    """With a limit of a nanosecond a wait that takes some microseconds is one that runs out: the tensor cores' warps wait for
    probabilities while the others add a step with undefined values key by key.  What was under way lands, the status says
    so, and the next call is as any other."""
    Hq, Hkv, hd = heads
    starts, lens, table, n_pages = _tables(seqs, seed=33)
    n = int(starts[-1])
    g = torch.Generator(device="cuda").manual_seed(34)
    pool = torch.randn((n_pages, Hkv, 2, 16, hd), generator=g, device="cuda").bfloat16()
    for s, (new, kv) in enumerate(seqs):
        for t in (kv - 1, kv - new // 2):                    # behind some row of the chunk
            pool[int(table[s, t // 16]), :, 1, t % 16, ::7] = float("nan")
    q = torch.randn((n, Hq, hd), generator=g, device="cuda").bfloat16()
    chunks = _batch(B, starts, lens, table, n, max(c for c, _ in seqs))
    good = B.echo_chunk_attention(chunks, q, pool)
    chunks.check()
    try:
        B.echo_debug_chunk_wait_limit(1)
        for _ in range(5):
            B.echo_chunk_attention(chunks, q, pool)
            with pytest.raises(B.EchoError, match="ECHO_ERR_TIMEOUT"):
                chunks.check()
    finally:
        B.echo_debug_chunk_wait_limit(0)
    for _ in range(3):
        assert torch.equal(torch.nan_to_num(B.echo_chunk_attention(chunks, q, pool)), torch.nan_to_num(good))
    chunks.check()
    with pytest.raises(B.EchoError, match="ECHO_ERR_INVALID"):
        B.echo_debug_chunk_wait_limit(1_000_000_001)
