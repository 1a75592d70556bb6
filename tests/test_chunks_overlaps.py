"""Arrays that a call of the caller's paged cache writes and that lie in its tables or status are refused on the host (no GPU
needed).  Addresses here are numbers that nothing reads."""
import pytest

from test_oracle_chunks import INVALID, P, _append, _attend, _chunks, lib  # noqa: F401

FAR = {"row_starts": 4096 * P, "kv_lens": 4097 * P, "page_table": 4098 * P, "status": 4099 * P}
SIZES = {"row_starts": 12, "kv_lens": 8, "page_table": 32, "status": 4}       # of 2 sequences of 4 pages


# what the default calls write, and its bytes: 7 pages of 2 heads of 128, 5 rows of 4 heads of 128, a workspace
@pytest.mark.parametrize("table", FAR)
@pytest.mark.parametrize("call,start,size", [
    (_append, 64 * P, 7 * 2 * 2 * 16 * 128 * 2), (_append, 32 * P, 5 * 4 * 128 * 2), (_attend, 32 * P, 5 * 4 * 128 * 2), (_attend, 512 * P, None),
])
def test_written_arrays_in_the_tables(lib, call, start, size, table):  # noqa: F811
    if size is None:
        size = lib.lib.echo_chunk_attention_workspace_bytes(5, 4, 2, 128)
    for at in (start, start + size - 4, start - SIZES[table] + 4):
        assert call(lib, _chunks(lib, **dict(FAR, **{table: at}))) == INVALID, at


@pytest.mark.parametrize("at", ["row_starts", "kv_lens", "page_table"])
def test_a_status_in_the_tables(lib, at):  # noqa: F811
    f = dict(FAR, status=FAR[at] + SIZES[at] - 4)
    assert _append(lib, _chunks(lib, **f)) == INVALID and _attend(lib, _chunks(lib, **f)) == INVALID


def test_a_status_in_what_is_read(lib):  # noqa: F811
    for at in (P, 2 * P, 3 * P):                             # q, k, v
        assert _append(lib, _chunks(lib, **dict(FAR, status=at))) == INVALID
    for at in (P, 64 * P):                                   # q, the pool
        assert _attend(lib, _chunks(lib, **dict(FAR, status=at))) == INVALID
