"""GPU parity of the caller's paged cache: echo_append_kv and echo_chunk_attention against the fp64 oracle.

Bounds are sums of roundings on the same (already rounded) inputs; e = 2^-24 is half a step of fp32, h half a step of
the cache's format (bf16 2^-8, half 2^-11).

  rotation   the angle's fraction of a turn is rounded to fp32 (at most 2^-26 of a turn, 2^-23.3 rad), sine and cosine
             are good to one step (2^-24), two products and a sum round three times: at most 2^-22 (|a| + |b|), then h
             of the result
  attention  a score of sum |q||k| / sqrt(hd) = z is a sum of hd products in fp32, in the tensor cores' order and
             truncated (2 e each), scaled and exponentiated (8 steps): d = 2 e (hd + 8) z relative in a probability, in
             numerator and denominator; probabilities are rounded to the format (h relative; in half, 2^-25 of the
             row's largest where they are below its normal numbers), products summed over n keys in fp32 (2 e n)
"""
import numpy as np
import pytest
import torch

from oracle import chunks as K

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def B():
    from paper_2602_02192_b200 import binding
    return binding


def _tables(seqs, extra_pages=2, seed=0, width=0):
    """row_starts, kv_lens, page_table (pages in random order, garbage behind a sequence's last) and the pages needed.
    seqs: (new tokens, keys once they are appended)."""
    rng = np.random.default_rng(seed)
    starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
    lens = np.array([kv for _, kv in seqs], dtype=np.int32)
    count = [-(-kv // 16) for _, kv in seqs]
    n_pages = sum(count) + extra_pages
    order, at = rng.permutation(n_pages).astype(np.int32), 0
    table = np.full((len(seqs), max(max(count), 1, width)), -7, dtype=np.int32)
    table[:, ::2] = 2 ** 30
    for s, c in enumerate(count):
        table[s, :c] = order[at:at + c]
        at += c
    return starts, lens, table, n_pages


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _batch(B, starts, lens, table, rows, longest):
    return B.KVChunks(_dev(starts), _dev(lens), _dev(table), rows, longest)


def _f64(x):
    return x.double().cpu().numpy()


def _check_attention(got, want, spread, scores, lens_by_row, v_top, dtype, hd):
    h = HALF_STEP[dtype]
    n = lens_by_row[:, None, None]
    d = 2 * E * (hd + 8) * scores[:, :, None]
    tol = h * np.abs(want) + (1 + h) * spread * (h + 2 * d + 2 * E * (n + 16)) + TINY[dtype]
    if dtype == torch.float16:
        tol = tol + n * 2.0 ** -25 * v_top
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5], tol[bad][:5])


# (new tokens, keys): one token and none, pages that end inside and at a tile, rows over several tiles, long caches
RAGGED = [(1, 1), (5, 5), (0, 33), (1, 128), (17, 128), (3, 129), (130, 130), (1, 1001), (33, 257), (2, 16), (1, 17)]
SHAPES = [(4, 2, 64), (32, 8, 128), (10, 2, 64), (3, 1, 128), (16, 16, 64), (7, 1, 128), (64, 8, 128)]


# ---- append ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("given", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,cut,offset", [((4, 2, 64), 0, 0), ((32, 8, 128), 1, 0), ((10, 2, 64), 1, 1), ((3, 1, 128), 0, 3),
                                              ((71, 1, 64), 1, 0)])
def test_append(B, given, cache, heads, cut, offset):
    Hq, Hkv, hd = heads
    seqs = RAGGED + [(2, 100003)]                        # a far position
    starts, lens, table, n_pages = _tables(seqs, seed=Hq)
    n, spare = int(starts[-1]), 6
    rng = np.random.default_rng(5)
    # cuts of one projection's rows, or arrays of their own; offset elements into their storage
    width, sizes = (Hq + 2 * Hkv) * hd, (Hq * hd, Hkv * hd, Hkv * hd)
    store = _dev(rng.normal(size=(n + spare) * (width + cut * 3 * offset) + offset)).to(given)
    whole = store[offset:].view(n + spare, -1)[:, :width]
    q, k, v = (x.view(n + spare, -1, hd) for x in whole.split(sizes, dim=1)) if cut else \
        (x.contiguous().view(n + spare, -1, hd) for x in whole.split(sizes, dim=1))
    pool = _dev(rng.normal(size=(n_pages, Hkv, 2, 16, hd))).to(cache)
    out = torch.full((n + spare, Hq, hd), 7.0, dtype=cache, device="cuda")
    before, theta = _f64(pool), 5e5
    chunks = _batch(B, starts, lens, table, n + spare, 130)
    B.echo_append_kv(chunks, q, k, v, pool, theta, out=out)
    chunks.check()
    q64, k64, v64 = _f64(q), _f64(k), _f64(v)
    want_pool, want_q = K.append(before, q64, k64, v64, starts, lens, table, theta)
    assert torch.all(out[n:] == 7.0)

    def close(got, want, x):
        half = hd // 2
        size = np.abs(x[..., :half]) + np.abs(x[..., half:])
        size = np.concatenate([size, size], axis=-1)
        assert np.all(np.abs(got - want) <= HALF_STEP[cache] * np.abs(want) + 2.0 ** -22 * (1 + HALF_STEP[cache]) * size + TINY[cache])

    close(_f64(out)[:n], want_q[:n], q64[:n])
    got = _f64(pool)
    mine = np.zeros((n_pages, 16), dtype=bool)
    for s, row, t in K.positions(starts, lens):
        page, slot = table[s, t // 16], t % 16
        mine[page, slot] = True
        close(got[page, :, 0, slot], want_pool[page, :, 0, slot], k64[row])
        assert np.array_equal(got[page, :, 1, slot], _f64(v[row].to(cache)))
    assert np.array_equal(got.transpose(0, 3, 1, 2, 4)[~mine], before.transpose(0, 3, 1, 2, 4)[~mine])      # nothing else is touched


def test_append_without_queries_in_place_and_far(B):
    Hq, Hkv, hd = 4, 2, 128
    starts, lens = np.array([0, 3], np.int32), np.array([2 ** 24 + 5], np.int32)
    table = np.zeros((1, (2 ** 24 + 5) // 16 + 1), np.int32)
    table[0, 2 ** 20:] = 1
    rng = np.random.default_rng(6)
    k, v, q = (_dev(rng.normal(size=(3, H, hd))).bfloat16() for H in (Hkv, Hkv, Hq))
    pools = [torch.zeros((2, Hkv, 2, 16, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    chunks = _batch(B, starts, lens, table, 3, 3)
    assert B.echo_append_kv(chunks, None, k, v, pools[0], 1e4) is None
    turned = B.echo_append_kv(chunks, q, k, v, pools[1], 1e4)
    kept = q.clone()
    assert B.echo_append_kv(chunks, q, k, v, pools[1], 1e4, out=q) is q and torch.equal(q, turned)
    chunks.check()
    assert torch.equal(pools[0], pools[1])
    _, want = K.append(_f64(pools[0]), _f64(kept), _f64(k), _f64(v), starts, lens, table, 1e4)
    size = np.abs(_f64(kept)).max()
    # at 2^24 the 64-bit product itself is off by 2^-53 of 2^24 / 2 pi turns: nothing beside the fp32 rounding
    assert np.all(np.abs(_f64(turned) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * 2.02 * size)


def test_append_many_rows(B):
    """Eight rows a CTA, rows that end inside one."""
    Hq, Hkv, hd, rows = 8, 2, 64, 20011
    seqs = [(5000, 5100), (1, 9), (0, 4), (9999, 9999), (5011, 8000)]
    starts, lens, table, n_pages = _tables(seqs)
    g = torch.Generator(device="cuda").manual_seed(1)
    whole = torch.randn((rows, (Hq + 2 * Hkv) * hd), generator=g, device="cuda")
    q, k, v = (x.view(rows, -1, hd) for x in whole.split((Hq * hd, Hkv * hd, Hkv * hd), dim=1))
    pool = torch.zeros((n_pages, Hkv, 2, 16, hd), dtype=torch.float16, device="cuda")
    chunks = _batch(B, starts, lens, table, rows, 9999)
    out = B.echo_append_kv(chunks, q, k, v, pool, 1e4)
    chunks.check()
    _, want = K.append(_f64(pool), _f64(q), _f64(k), _f64(v), starts, lens, table, 1e4)
    size = np.abs(_f64(q)).max(axis=2, keepdims=True) * 2
    assert np.all(np.abs(_f64(out) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -22 * 1.01 * size + 2.0 ** -25)
    t = torch.tensor([(table[s, p // 16], p % 16, r) for s, r, p in K.positions(starts, lens)], device="cuda")
    assert torch.equal(pool[t[:, 0], :, 1, t[:, 1]], v[t[:, 2]].half())


# ---- attention ------------------------------------------------------------------------------------
def _attention_case(B, heads, dtype, seqs, seed=0, pad=0, spare=3, q_size=1.0, spoil=None, longest=None):
    """Runs the call on a pool that holds NaN wherever no key of the sequences is; compares with the oracle."""
    Hq, Hkv, hd = heads
    starts, lens, table, n_pages = _tables(seqs, seed=seed)
    n = int(starts[-1])
    rng = np.random.default_rng(seed + 1)
    kv = rng.normal(size=(n_pages, Hkv, 2, 16, hd))
    filled = np.full(kv.shape, np.nan)
    for s, (_, keys) in enumerate(seqs):
        for t0 in range(0, keys, 16):
            here = min(16, keys - t0)
            filled[table[s, t0 // 16], :, :, :here] = kv[table[s, t0 // 16], :, :, :here]
    if spoil is not None:
        spoil(filled, starts, lens, table)
    pool = _dev(filled).to(dtype)
    store = torch.zeros((n + spare, Hq * hd + pad), dtype=dtype, device="cuda")
    q = store[:, :Hq * hd].view(n + spare, Hq, hd)
    q.copy_(_dev(rng.normal(size=q.shape) * q_size))
    out = torch.full((n + spare, Hq, hd), 7.0, dtype=dtype, device="cuda")
    chunks = _batch(B, starts, lens, table, n + spare, longest or max(max(s[0] for s in seqs), 1))
    got = B.echo_chunk_attention(chunks, q, pool, out=out)
    chunks.check()
    assert torch.all(got[n:] == 7.0)
    pool64, q64 = _f64(pool), _f64(q)
    want, spread, scores = K.attend(pool64, q64, starts, lens, table, np.full(q64.shape, 7.0))
    keys = np.zeros(n + spare)
    for s, row, t in K.positions(starts, lens):
        keys[row] = max(t + 1, 0)
    return _f64(got), want, spread, scores, keys, np.abs(kv).max()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads", SHAPES)
def test_attention_of_ragged_chunks(B, heads, dtype):
    got, want, spread, scores, keys, top = _attention_case(B, heads, dtype, RAGGED, seed=heads[0], pad=8 * (heads[0] % 3))
    _check_attention(got, want, spread, scores, keys, top, dtype, heads[2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,seqs", [
    ((32, 8, 128), [(1, 9000)]),                              # one row, many tiles: the cache is cut and joined
    ((2, 1, 64), [(1, 33333)]),
    ((8, 1, 128), [(40, 7003)]),
    ((4, 4, 128), [(300, 2500), (1, 1), (259, 259)]),         # no sharing: whole tiles of rows
    ((128, 1, 64), [(5, 700), (2, 2)]),                       # a row tile is one token
    ((48, 1, 128), [(9, 300)]),                               # two tokens a row tile, rows of it unused
    ((12, 2, 64), [(700, 1024), (64, 640)]),
    ((4, 2, 64), [(1, n) for n in range(1, 290, 7)]),         # many sequences of one token
    ((16, 8, 128), [(n, 2 * n) for n in range(1, 60)]),
    ((8, 8, 128), [(1, 20000)] * 6 + [(2, 17)]),              # dozens of tiles in a row for each CTA
    ((16, 8, 128), [(130, 9300), (1, 9000), (67, 6500)]),
    ((8, 8, 64), [(1, 30000)] * 5 + [(140, 4000)]),
    ((64, 8, 128), [(130, 130), (70, 200)] * 5),             # many short items
    ((32, 8, 128), [(16, 300), (3, 40), (1, 5000), (16, 16)]),        # no more than 64 rows to an item
    ((48, 1, 128), [(1, 600), (1, 1)]),                       # the same, one token of 48 heads
    ((2, 1, 64), [(1, 1 + s % 50) if s % 7 else (0, 9) for s in range(1500)]),      # more sequences than a CTA has threads
    ((4, 2, 64), [(0, 3)] * 1300 + [(40, 170), (1, 300)]),
])
def test_attention_of_long_caches_and_odd_groups(B, heads, seqs, dtype):
    got, want, spread, scores, keys, top = _attention_case(B, heads, dtype, seqs, seed=3)
    _check_attention(got, want, spread, scores, keys, top, dtype, heads[2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [12.0, 1e-3])
def test_attention_of_peaked_and_flat_rows(B, dtype, size):
    got, want, spread, scores, keys, top = _attention_case(B, (8, 2, 128), dtype, [(1, 3000), (200, 900), (7, 7)], seed=4, q_size=size)
    _check_attention(got, want, spread, scores, keys, top, dtype, 128)


def test_rows_that_see_nothing_are_zero(B):
    """Chunks longer than their caches: positions below 0; no keys at all."""
    seqs = [(5, 2), (3, 0), (200, 70), (1, 1)]
    got, want, spread, scores, keys, top = _attention_case(B, (4, 2, 64), torch.bfloat16, seqs, seed=5)
    assert np.all(got[:3] == 0) and np.all(got[5:8] == 0) and np.all(got[8:138] == 0)
    _check_attention(got, want, spread, scores, keys, top, torch.bfloat16, 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("what", [0, 1])                     # in a key, in a value
def test_what_a_row_does_not_see_has_no_part_in_it(B, dtype, value, what):
    """Undefined keys and values behind a row's position (of later tokens of its own chunk): the rows before them are
    what they would be without, the rows behind are undefined where the formula is."""
    seqs = [(40, 300), (150, 150), (1, 40)]
    at = [(0, 280), (1, 60), (1, 149)]                       # sequence, position

    def spoil(kv, starts, lens, table):
        for s, t in at:
            kv[table[s, t // 16], 1, what, t % 16, 5] = value

    got, want, spread, scores, keys, top = _attention_case(B, (8, 2, 64), dtype, seqs, seed=6, spoil=spoil)
    fine = np.isfinite(want)
    assert not fine.all() and np.array_equal(np.isfinite(got), fine)
    if what == 1:                                            # p v is NaN or an infinity of v's sign
        assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
    z = np.where(np.isfinite(scores), scores, 0)
    _check_attention(np.where(fine, got, 0), np.where(fine, want, 0), np.where(fine, spread, 0), z, keys, top, dtype, 64)


@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("longest", [None, 200])             # rows in tiles of 64, of 128
def test_an_undefined_query_spoils_its_row_alone(B, value, longest):
    Hq, Hkv, hd = 8, 2, 64
    seqs = [(3, 700), (9, 9)] if longest is None else [(3, 700), (150, 300)]
    starts, lens, table, n_pages = _tables(seqs, seed=11)
    n = int(starts[-1])
    rng = np.random.default_rng(12)
    pool = _dev(rng.normal(size=(n_pages, Hkv, 2, 16, hd))).bfloat16()
    q = _dev(rng.normal(size=(n, Hq, hd))).bfloat16()
    chunks = _batch(B, starts, lens, table, n, longest or 9)
    q[1, 5, 3], q[5, 0, 0] = value, value
    got = _f64(B.echo_chunk_attention(chunks, q, pool))
    chunks.check()
    spoiled = np.zeros((n, Hq), dtype=bool)
    spoiled[1, 5] = spoiled[5, 0] = True
    assert np.isnan(got[spoiled]).all()
    q[1, 5, 3], q[5, 0, 0] = 0, 0
    want, spread, scores = K.attend(_f64(pool), _f64(q), starts, lens, table, np.zeros(q.shape))
    got[spoiled], want[spoiled] = 0, 0       # (the other rows of a warp may round their probabilities at other references)
    keys = np.zeros(n)
    for s, row, t in K.positions(starts, lens):
        keys[row] = t + 1
    _check_attention(got, want, spread, scores, keys, 8.0, torch.bfloat16, hd)


def test_bad_pages_and_lengths_are_reported(B):
    Hq, Hkv, hd = 8, 2, 128
    seqs = [(2, 40), (3, 500), (1, 200), (4, 90)]
    starts, lens, table, n_pages = _tables(seqs)
    n = int(starts[-1])
    g = torch.Generator(device="cuda").manual_seed(2)
    pool = torch.randn((n_pages, Hkv, 2, 16, hd), generator=g, device="cuda").bfloat16()
    q = torch.randn((n, Hq, hd), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((n, Hkv, hd), generator=g, device="cuda").bfloat16() for _ in range(2))
    good = B.echo_chunk_attention(_batch(B, starts, lens, table, n, 4), q, pool)
    for page in (-1, n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.copy()
        t[1, 3] = page                                       # a page in the middle of sequence 1's cache
        chunks = _batch(B, starts, lens, t, n, 4)
        out = B.echo_chunk_attention(chunks, q, pool)
        with pytest.raises(B.EchoError, match="ECHO_ERR_DEVICE_CHECK"):
            chunks.check()
        chunks.check()                                       # zeroed
        assert torch.isnan(out[2:5]).all() and torch.equal(out[:2], good[:2]) and torch.equal(out[5:], good[5:])
        t = table.copy()
        t[1, 31] = page                                      # the page that its new tokens go to
        chunks, after = _batch(B, starts, lens, t, n, 4), pool.clone()
        turned = B.echo_append_kv(chunks, q, k, v, after, 1e4)
        with pytest.raises(B.EchoError, match="a page id"):
            chunks.check()
        whole = pool.clone()
        assert torch.equal(turned, B.echo_append_kv(_batch(B, starts, lens, table, n, 4), q, k, v, whole, 1e4))
        assert torch.equal(after[table[1, 31]], pool[table[1, 31]])
        keep = torch.arange(n_pages, device="cuda") != int(table[1, 31])
        assert torch.equal(after[keep], whole[keep])
    # lengths: a chunk longer than the batch says, a cache longer than the table, a decreasing start, a negative length
    for change in (dict(longest=3), dict(lens=(2, 16 * table.shape[1] + 1)), dict(lens=(2, -1)), dict(starts=(3, 4)), dict(starts=(4, n + 1))):
        st, ln = starts.copy(), lens.copy()
        if "lens" in change:
            ln[change["lens"][0]] = change["lens"][1]
        if "starts" in change:
            st[change["starts"][0]] = change["starts"][1]
        chunks = _batch(B, st, ln, table, n, change.get("longest", 4))
        out = B.echo_chunk_attention(chunks, q, pool, out=torch.full_like(q, 7.0))
        with pytest.raises(B.EchoError, match="lengths"):
            chunks.check()
        after = pool.clone()
        turned = B.echo_append_kv(chunks, q, k, v, after, 1e4, out=torch.full_like(q, 7.0))
        with pytest.raises(B.EchoError, match="lengths"):
            chunks.check()
        # sequence 0 is untouched by any of these; rows that only sequences out of the limits name are left as they were
        assert torch.equal(out[:2], good[:2])
        fine, named = np.zeros(n + 9, dtype=bool), np.zeros(n + 9, dtype=bool)
        for s in range(4):
            r0, r1 = int(st[s]), int(st[s + 1])
            bad = r1 < r0 or r1 > n or r1 - r0 > chunks.max_chunk or not 0 <= ln[s] <= 16 * table.shape[1]
            (named if bad else fine)[r0:r1] = True
        left = torch.from_numpy(np.flatnonzero((named & ~fine)[:n])).cuda()
        assert torch.all(out[left] == 7.0) and torch.all(turned[left] == 7.0)
    # a chunk longer than its cache is not appended
    chunks, after = _batch(B, starts, np.array([1, 500, 200, 90], np.int32), table, n, 4), pool.clone()
    turned = B.echo_append_kv(chunks, q, k, v, after, 1e4, out=torch.full_like(q, 7.0))
    with pytest.raises(B.EchoError, match="lengths"):
        chunks.check()
    assert torch.all(turned[:2] == 7.0) and torch.equal(after[table[0, :3]], pool[table[0, :3]])


def test_offsets_past_32_bits(B):
    """Pages more than 2^31 elements (and 4 GB) into the pool."""
    Hq, Hkv, hd = 8, 8, 128
    n_pages = 2 ** 32 // (Hkv * 2 * 16 * hd * 2) + 2 ** 31 // (Hkv * 2 * 16 * hd) + 40
    pool = torch.empty((n_pages, Hkv, 2, 16, hd), dtype=torch.bfloat16, device="cuda")
    seqs = [(20, 300), (1, 150)]
    starts, lens, table, need = _tables(seqs, extra_pages=0)
    small = torch.empty((need, Hkv, 2, 16, hd), dtype=torch.bfloat16, device="cuda").normal_()
    far = n_pages - need
    pool[far:] = small
    k, v, q = (torch.randn((21, H, hd), device="cuda") for H in (Hkv, Hkv, Hq))
    here, there = _batch(B, starts, lens, table, 21, 20), _batch(B, starts, lens, table + far, 21, 20)
    a, b = B.echo_append_kv(here, q, k, v, small), B.echo_append_kv(there, q, k, v, pool)
    assert torch.equal(a, b) and torch.equal(pool[far:], small)
    assert torch.equal(B.echo_chunk_attention(here, a, small), B.echo_chunk_attention(there, a, pool))
    here.check()
    there.check()


def test_equal_inputs_give_equal_outputs_on_any_stream(B):
    """Twice, on two streams at once, and in a graph whose tables change between replays."""
    Hq, Hkv, hd = 32, 8, 128
    seqs = [(1, 4000), (65, 900), (0, 10), (7, 2049), (130, 131)]
    starts, lens, table, n_pages = _tables(seqs, extra_pages=0, width=300)
    n = int(starts[-1])
    g = torch.Generator(device="cuda").manual_seed(3)
    pool = torch.randn((n_pages, Hkv, 2, 16, hd), generator=g, device="cuda").bfloat16()
    q = torch.randn((n, Hq, hd), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((n, Hkv, hd), generator=g, device="cuda") for _ in range(2))
    qf = q.float()
    chunks = _batch(B, starts, lens, table, n, 130)
    first_pool = pool.clone()
    turned = B.echo_append_kv(chunks, qf, k, v, first_pool)
    first = B.echo_chunk_attention(chunks, turned, first_pool)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            p = pool.clone()
            t = B.echo_append_kv(chunks, qf, k, v, p)
            got.append((p, t, [B.echo_chunk_attention(chunks, t, p) for _ in range(3)]))
    torch.cuda.synchronize()
    for p, t, outs in got:
        assert torch.equal(p, first_pool) and torch.equal(t, turned) and all(torch.equal(o, first) for o in outs)
    # captured, replayed, and replayed after the tables' contents have changed: as eager calls on these tables
    p, out = pool.clone(), torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t = B.echo_append_kv(chunks, qf, k, v, p)
        B.echo_chunk_attention(chunks, t, p, out=out)
    for _ in range(2):
        graph.replay()
    assert torch.equal(out, first) and torch.equal(p, first_pool)
    row_starts, kv_lens, page_table = chunks._keep
    kv_lens.copy_(_dev(np.array([3000, 80, 10, 1111, 131], np.int32)))
    row_starts.copy_(_dev(np.array([0, 2, 66, 70, 73, n], np.int32)))
    graph.replay()
    eager_pool = first_pool.clone()
    t2 = B.echo_append_kv(chunks, qf, k, v, eager_pool)
    want = B.echo_chunk_attention(chunks, t2, eager_pool)
    chunks.check()
    assert torch.equal(out, want) and torch.equal(p, eager_pool)


def test_a_conversation_in_pieces_is_the_conversation_at_once(B):
    """Prompt, single tokens, a tool's answer, single tokens: appended and attended piece by piece, against the oracle's
    attention over the whole, and echo_decode_attention on the same pages."""
    Hq, Hkv, hd, dtype = 8, 2, 128, torch.bfloat16
    pieces = [37, 1, 1, 300, 1, 64, 1]
    total = sum(pieces)
    rng = np.random.default_rng(8)
    q, k, v = (_dev(rng.normal(size=(2, total, H, hd))).float() for H in (Hq, Hkv, Hkv))
    width = -(-total // 16)
    table = rng.permutation(2 * width).reshape(2, width).astype(np.int32)
    pool = torch.full((2 * width, Hkv, 2, 16, hd), float("nan"), dtype=dtype, device="cuda")
    at, outs, turned_all = 0, [], []
    for n in pieces:
        starts, lens = np.array([0, n, 2 * n], np.int32), np.array([at + n] * 2, np.int32)
        chunks = _batch(B, starts, lens, table, 2 * n, n)
        cut = [x[:, at:at + n].reshape(2 * n, -1, hd) for x in (q, k, v)]
        turned = B.echo_append_kv(chunks, *cut, pool, 1e4)
        outs.append(B.echo_chunk_attention(chunks, turned, pool).view(2, n, Hq, hd))
        turned_all.append(turned.view(2, n, Hq, hd))
        chunks.check()
        at += n
    got, turned = torch.cat(outs, dim=1), torch.cat(turned_all, dim=1)
    lens = np.array([total] * 2, np.int32)
    starts = np.array([0, total, 2 * total], np.int32)
    want, spread, scores = K.attend(np.nan_to_num(_f64(pool)), _f64(turned).reshape(-1, Hq, hd), starts, lens, table, np.zeros((2 * total, Hq, hd)))
    keys = np.tile(np.arange(1, total + 1), 2)
    _check_attention(_f64(got).reshape(-1, Hq, hd), want, spread, scores, keys, 8.0, dtype, hd)
    pool = torch.nan_to_num(pool)
    last = B.echo_decode_attention(turned[:, -1].contiguous(), pool, _dev(table), _dev(lens - 1), torch.zeros(2, dtype=torch.int32, device="cuda"), 2, 1)
    h = HALF_STEP[dtype]
    rows = [total - 1, 2 * total - 1]
    assert np.all(np.abs(_f64(last) - want[rows]) <= 2 * h * np.abs(want[rows]) + 4 * h * spread[rows])


def test_a_decoder_layer_by_layer_scores_as_the_engine_does(B):
    """Two layers run by a caller on the library's own pieces: projections, append, attention over a cache that takes the
    prompt in two pieces and the response in one, log-probabilities; against the fp64 decoder, with the tolerance that the
    engine's own scores have (5e-2), and against echo_score (both: twice that)."""
    from oracle import decoder
    from paper_2602_02192_b200 import synth
    wl = synth.WORKLOADS["tiny"]
    S, P, G, Lp, T = wl.shape, 2, 1, 45, 20
    w_t = synth.make_weights(S, wl.weight_seed)
    w = {k: ([x.cuda() for x in v] if isinstance(v, list) else v.cuda()) for k, v in w_t.items()}
    prompts = synth.make_prompts(P, Lp, S.vocab, wl.prompt_seed)
    rng = np.random.default_rng(9)
    response = rng.integers(0, S.vocab, size=(P, T)).astype(np.int32)
    whole = np.concatenate([prompts, response], axis=1)
    Hq, Hkv, hd = S.n_q_heads, S.n_kv_heads, S.head_dim
    width = -(-(Lp + T) // 16)
    table = rng.permutation(P * width).reshape(P, width).astype(np.int32)
    pools = [torch.full((P * width, Hkv, 2, 16, hd), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(S.n_layers)]

    def norm(x, gain):
        return (x * torch.rsqrt(x.pow(2).mean(dim=1, keepdim=True) + S.rms_eps) * gain.float()).bfloat16()

    def advance(at, n):
        """Feeds positions at .. at + n - 1 of every sequence; the residual stream of these rows."""
        chunks = _batch(B, np.arange(P + 1, dtype=np.int32) * n, np.full(P, at + n, np.int32), table, P * n, n)
        x = w["embed"][torch.from_numpy(whole[:, at:at + n].reshape(-1).astype(np.int64)).cuda()].float()
        for l in range(S.n_layers):
            h = norm(x, w["attn_norm"][l])
            qkv = B.echo_gemm_bf16(h, torch.cat([w["wq"][l], w["wk"][l], w["wv"][l]]))
            q, k, v = (y.view(P * n, -1, hd) for y in qkv.split((Hq * hd, Hkv * hd, Hkv * hd), dim=1))
            q = B.echo_append_kv(chunks, q, k, v, pools[l], S.rope_theta)
            o = B.echo_chunk_attention(chunks, q, pools[l])
            x = B.echo_gemm_bf16(o.view(P * n, Hq * hd), w["wo"][l], epilogue=1, Y=x)
            act = B.echo_gemm_bf16(norm(x, w["mlp_norm"][l]), torch.cat([w["w_gate"][l], w["w_up"][l]]), epilogue=2)
            x = B.echo_gemm_bf16(act, w["w_down"][l], epilogue=1, Y=x)
        chunks.check()
        return x.view(P, n, -1)

    advance(0, 30)
    x = torch.cat([advance(30, Lp - 30)[:, -1:], advance(Lp, T - 1)], dim=1)     # what predicts the response
    logits = B.echo_gemm_bf16(norm(x.reshape(P * T, -1), w["final_norm"]), w["lm_head"])
    got = B.echo_token_logprobs(logits, torch.from_numpy(response.reshape(-1)).cuda())[0].view(P, T).cpu().numpy()
    dims = decoder.ModelDims(S.n_layers, S.d_model, Hq, Hkv, hd, S.d_ff, S.vocab, S.rms_eps, S.rope_theta)
    weights = decoder.Weights(synth.weights_to_bits(w_t))
    for p in range(P):
        want = decoder.score_forced(dims, weights, prompts[p], response[p], 1.0, 0, p).logprob_given
        assert np.all(np.abs(got[p] - want) <= 5e-2)
    eng = B.Engine(B.make_config(S, P, G, Lp, T))
    eng.echo_load_policy(w, 1)
    lp, _ = eng.echo_score(torch.from_numpy(prompts).cuda(), [Lp] * P, torch.from_numpy(response[:, None]).cuda(), 1.0)
    eng.echo_sync()
    assert np.all(np.abs(lp[:, 0].cpu().numpy() - got) <= 1e-1)
    eng.close()


@pytest.mark.parametrize("S", [0, 3])
def test_a_batch_without_new_tokens(B, S):
    chunks = B.KVChunks(torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.full((S,), 5, dtype=torch.int32, device="cuda"),
                        torch.zeros((S, 1), dtype=torch.int32, device="cuda"), 0, 0)
    pool = torch.ones((2, 2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    q, k, v = (torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    assert B.echo_append_kv(chunks, q, k, v, pool).shape == q.shape
    assert B.echo_append_kv(chunks, None, k, v, pool) is None
    assert B.echo_chunk_attention(chunks, q, pool).shape == q.shape
    chunks.check()
    assert bool((pool == 1).all())


@pytest.mark.parametrize("n", [1, 66])
def test_many_small_probabilities_beside_a_large_one(B, n):
    """One key whose score is 17.6 above those of all others: each of these has a probability of 2^-25.4, below half of
    half precision's smallest number, and together they are all that the result holds.  Relative to 2^6 for the largest
    they are rounded by at most 2^-31 of it each; everything else is as in the attention's bound above."""
    S, kv, hd = 150, 30000, 64
    pages = -(-kv // 16)
    pool = torch.zeros((pages, 1, 2, 16, hd), dtype=torch.float16, device="cuda")
    pool[:, :, 1] = 1
    q = torch.zeros((S * n, 2, hd), dtype=torch.float16, device="cuda")
    q[..., 0] = pool[0, 0, 0, 0, 0] = 11.866
    pool[0, 0, 1, 0] = 0
    starts, lens = np.arange(S + 1, dtype=np.int32) * n, np.full(S, kv, np.int32)
    table = np.tile(np.random.default_rng(0).permutation(pages).astype(np.int32), (S, 1))
    table[:, np.flatnonzero(table[0] == 0)[0]], table[:, 0] = table[0, 0], 0          # the large one first
    chunks = _batch(B, starts, lens, table, S * n, n)
    got = _f64(B.echo_chunk_attention(chunks, q, pool)).reshape(S, n, 2, hd)
    chunks.check()
    want, *_ = K.attend(_f64(pool), _f64(q[:n]), starts[:2], lens[:1], table[:1], np.zeros((n, 2, hd)))
    z = 11.866 ** 2 / 8
    bound = np.abs(want) * (2 * HALF_STEP[torch.float16] + 2 * E * kv + 4 * E * (hd + 8) * z) + kv * TINY[torch.float16] / 64
    assert np.all(want > 6e-4) and np.all(np.abs(got - want[None]) <= bound[None])
