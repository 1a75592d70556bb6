"""Pins of the oracle of the caller's paged cache, and the refusals of the library's entry points (no GPU needed)."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import chunks as K


# ---- oracle ---------------------------------------------------------------------------------------
def test_rotation_angles_and_relative_positions():
    x = np.zeros((1, 4))
    x[0, 0] = 1.0                                       # pair (0, 2) turns by the position itself, (1, 3) by t / 10
    assert np.allclose(K.rotate(x, 3, 100.0), [[math.cos(3), 0, math.sin(3), 0]], atol=1e-15)
    x[0] = [0, 0, 0, 1.0]
    assert np.allclose(K.rotate(x, 5, 100.0), [[0, -math.sin(0.5), 0, math.cos(0.5)]], atol=1e-15)
    rng = np.random.default_rng(0)
    a, b = rng.normal(size=(1, 64)), rng.normal(size=(1, 64))
    d = [float((K.rotate(a, t + 7, 1e4) * K.rotate(b, t, 1e4)).sum()) for t in (0, 11, 100000)]
    assert np.allclose(d, d[0], atol=1e-9)              # only the distance matters
    assert np.array_equal(K.rotate(a, 0, 1e4), a)


def test_append_goes_to_the_tables_places():
    rng = np.random.default_rng(1)
    pool = rng.normal(size=(6, 2, 2, 16, 8))
    starts, lens, table = [0, 3, 3, 4], [17, 5, 1], np.array([[4, 2], [0, 0], [5, 0]])
    q, k, v = rng.normal(size=(6, 4, 8)), rng.normal(size=(6, 2, 8)), rng.normal(size=(6, 2, 8))
    new, turned = K.append(pool, q, k, v, starts, lens, table, 1e4)
    places = [(4, 14, 0), (4, 15, 1), (2, 0, 2), (5, 0, 3)]            # page, slot, row
    for page, slot, row in places:
        assert np.array_equal(new[page, :, 1, slot], v[row])
    assert np.allclose(new[4, :, 0, 15], K.rotate(k[1], 15, 1e4)) and np.array_equal(new[5, :, 0, 0], k[3])
    changed = np.any(new != pool, axis=(1, 2, 4))
    assert sorted(zip(*np.nonzero(changed))) == sorted((p, s) for p, s, _ in places)
    assert np.array_equal(turned[4:], q[4:])


def test_attention_of_one_key_equal_keys_and_nothing():
    rng = np.random.default_rng(2)
    pool = rng.normal(size=(3, 1, 2, 16, 8))
    pool[1, 0, 0, :] = pool[1, 0, 0, 0]                  # equal keys: the mean of the values
    q = rng.normal(size=(4, 2, 8))
    out, spread, _ = K.attend(pool, q, [0, 1, 2, 4], [1, 16, 1], np.array([[0], [1], [2]]), np.full((4, 2, 8), 9.0))
    assert np.allclose(out[0], pool[0, 0, 1, 0]) and np.allclose(spread[0], np.abs(pool[0, 0, 1, 0]))
    assert np.allclose(out[1], pool[1, 0, 1].mean(axis=0))
    assert np.all(out[2] == 0) and np.allclose(out[3], pool[2, 0, 1, 0])      # two rows over one key: positions -1 and 0


def test_a_chunk_is_its_tokens_one_by_one():
    rng = np.random.default_rng(3)
    pool, q, table = rng.normal(size=(3, 2, 2, 16, 8)), rng.normal(size=(5, 6, 8)), np.array([[2, 0, 1]])
    whole, *_ = K.attend(pool, q, [0, 5], [39], table, np.zeros((5, 6, 8)))
    for i in range(5):
        one, *_ = K.attend(pool, q[i:i + 1], [0, 1], [35 + i], table, np.zeros((1, 6, 8)))
        assert np.allclose(one[0], whole[i], atol=1e-14)


# ---- refusals -------------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def lib():
    from paper_2602_02192_b200 import binding
    return binding


P = 1 << 20          # an address that nothing reads: every call below is refused on the host


def _chunks(lib, **change):
    f = dict(row_starts=P, kv_lens=P, page_table=P, status=P, n_seqs=2, n_rows=5, pt_width=4, max_chunk=5)
    f.update(change)
    return lib.EchoKVChunks(**f)


def _append(lib, chunks=None, **change):
    f = dict(q=P, k=2 * P, v=3 * P, in_format=2, q_stride=512, k_stride=256, v_stride=256, chunks=chunks or _chunks(lib), Hq=4,
             Hkv=2, hd=128, rope_theta=1e4, kv_pool=64 * P, n_pages=7, kv_format=0, out_q=32 * P, stream=None)
    f.update(change)
    f["chunks"] = C.byref(f["chunks"]) if isinstance(f["chunks"], C.Structure) else None
    return lib.lib.echo_append_kv(*f.values())


def _attend(lib, chunks=None, **change):
    f = dict(q=P, q_stride=512, kv_pool=64 * P, n_pages=7, format=0, chunks=chunks or _chunks(lib), Hq=4, Hkv=2, hd=128,
             workspace=512 * P, workspace_bytes=1 << 30, out=32 * P, stream=None)
    f.update(change)
    f["chunks"] = C.byref(f["chunks"]) if isinstance(f["chunks"], C.Structure) else None
    return lib.lib.echo_chunk_attention(*f.values())


INVALID, UNSUPPORTED = -1, -9


@pytest.mark.parametrize("call", [_append, _attend])
def test_batches_that_are_refused(lib, call):
    for change in (dict(row_starts=None), dict(kv_lens=None), dict(page_table=None), dict(status=None), dict(n_seqs=-1),
                   dict(n_rows=-1), dict(pt_width=0), dict(max_chunk=0), dict(kv_lens=P + 2)):
        assert call(lib, _chunks(lib, **change)) == INVALID, change
    assert call(lib, _chunks(lib, pt_width=(1 << 26) + 1)) == UNSUPPORTED
    assert call(lib, chunks=1) == INVALID                       # no batch
    assert call(lib, _chunks(lib, n_seqs=0)) == 0 and call(lib, _chunks(lib, n_rows=0)) == 0


@pytest.mark.parametrize("change", [dict(n_seqs=0), dict(n_rows=0)])
def test_a_batch_of_nothing_needs_no_arrays(lib, change):
    f = dict(row_starts=None, kv_lens=None, page_table=None, status=None, pt_width=0, max_chunk=0, **change)
    for q in (P, None):
        assert _append(lib, _chunks(lib, **f), q=q, k=None, v=None, out_q=q and 32 * P) == 0
        assert _attend(lib, _chunks(lib, **f), q=q, out=None, workspace=None, workspace_bytes=0) == 0
    assert _append(lib, _chunks(lib, **f), Hkv=0) == INVALID and _attend(lib, _chunks(lib, **f), q_stride=504) == INVALID
    f["max_chunk"] = -1
    assert _append(lib, _chunks(lib, **f)) == INVALID and _attend(lib, _chunks(lib, **f)) == INVALID


@pytest.mark.parametrize("call", [_append, _attend])
def test_shapes_and_pools_that_are_refused(lib, call):
    for change in (dict(Hkv=0), dict(Hq=5), dict(Hq=-2), dict(hd=0), dict(kv_pool=None), dict(kv_pool=64 * P + 8),
                   dict(n_pages=0)):
        assert call(lib, **change) == INVALID, change
    for hd in (32, 96, 256):
        assert call(lib, hd=hd, q_stride=4 * hd) == UNSUPPORTED


def test_appends_that_are_refused(lib):
    for change in (dict(k=None), dict(v=None), dict(q=None), dict(out_q=None), dict(Hq=0), dict(in_format=3), dict(in_format=-1),
                   dict(kv_format=2), dict(rope_theta=0.0), dict(rope_theta=-1.0), dict(rope_theta=math.inf),
                   dict(rope_theta=math.nan), dict(q_stride=511), dict(k_stride=255), dict(v_stride=255), dict(v_stride=-256),
                   dict(k_stride=(1 << 30) + 1), dict(q=P + 2), dict(out_q=32 * P + 8)):
        assert _append(lib, **change) == INVALID, change
    # arrays that overlap: the pool with an input or the output, the output with keys, queries not in place
    assert _append(lib, kv_pool=P) == INVALID and _append(lib, k=64 * P + 16) == INVALID
    assert _append(lib, out_q=64 * P) == INVALID and _append(lib, out_q=2 * P) == INVALID
    assert _append(lib, out_q=P) == INVALID                     # in place needs the cache's format
    assert _append(lib, in_format=0, out_q=P, q_stride=520) == INVALID          # and rows that lie as the output's do
    assert _append(lib, in_format=0, out_q=P + 16) == INVALID


def test_attention_that_is_refused(lib):
    for change in (dict(q=None), dict(out=None), dict(Hq=0), dict(format=2), dict(format=-1), dict(q_stride=504),
                   dict(q_stride=516), dict(q_stride=(1 << 30) + 8), dict(q=P + 8), dict(out=32 * P + 8), dict(workspace=None),
                   dict(workspace=512 * P + 8), dict(workspace_bytes=0)):
        assert _attend(lib, **change) == INVALID, change
    assert _attend(lib, out=P) == INVALID and _attend(lib, out=64 * P) == INVALID
    assert _attend(lib, workspace=32 * P) == INVALID and _attend(lib, workspace=P) == INVALID
    assert _attend(lib, workspace=64 * P) == INVALID
    assert _attend(lib, Hq=258, q_stride=258 * 128) == UNSUPPORTED              # 129 query heads to a kv head
    assert _attend(lib, n_pages=(1 << 25) + 1) == UNSUPPORTED
    need = lib.lib.echo_chunk_attention_workspace_bytes(5, 4, 2, 128)
    assert need > 0 and _attend(lib, workspace_bytes=need - 1) == INVALID
    for bad in ((0, 4, 2, 128), (5, 0, 2, 128), (5, 4, 0, 128), (5, 5, 2, 128), (5, 4, 2, 96)):
        assert lib.lib.echo_chunk_attention_workspace_bytes(*bad) == 0


def test_struct_layout_matches_the_header(tmp_path):
    import os
    import subprocess
    from paper_2602_02192_b200 import binding
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    names = [f for f, _ in binding.EchoKVChunks._fields_]
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "echo.h"\nint main(void) {\nprintf("%zu\\n", sizeof(echo_kv_chunks));\n' +
                   "\n".join(f'printf("%zu\\n", offsetof(echo_kv_chunks, {f}));' for f in names) + "\nreturn 0; }\n")
    subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    out = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    assert out == [C.sizeof(binding.EchoKVChunks)] + [getattr(binding.EchoKVChunks, f).offset for f in names]
