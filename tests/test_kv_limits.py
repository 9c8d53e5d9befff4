"""Limits of cached attention that include/moin.h names, and what the size of its scratch depends on (no GPU needed)."""
import pytest

from test_kv_refusals import NO_DEVICE, SHAPE, WORKSPACE, A, _kv, _tables, lib  # noqa: F401

AUTO, ROWS, TENSOR = 0, 1, 2


@pytest.fixture
def option(lib):  # noqa: F811
    yield lambda v: lib.lib().moin_set_option(1, v)
    lib.lib().moin_set_option(1, AUTO)


@pytest.mark.parametrize("R,rows,max_q,heads,kv_heads,status", [
    (65535, 65535, 1, 2, 2, NO_DEVICE), (65536, 65536, 1, 2, 2, SHAPE), (65536, 65536, 1, 2, 1, SHAPE),
    (1, 4, (1 << 20) - 1, 64, 1, NO_DEVICE), (1, 4, 1 << 20, 64, 1, SHAPE), (1, 4, 1 << 20, 128, 2, SHAPE), (1, 4, 1 << 20, 32, 1, NO_DEVICE)])
def test_most_requests_and_rows_of_a_request(lib, R, rows, max_q, heads, kv_heads, status):  # noqa: F811
    T = max(R, max_q)
    stride = heads * 64
    got = lib.lib().moin_kv_attention(_kv(lib, heads=kv_heads), _tables(lib, n_rows=rows), None, A, A, R, T, max_q, 16, A, stride, heads, 0.125,
                                      None, 0, A, stride, A, 1 << 40, None)
    assert got == status


def test_scratch_is_asked_for_under_the_option_of_the_call(lib, option):  # noqa: F811
    L = lib.lib()
    args = (4, 4 * 64, 64, 128, 8, 2, 64)        # R, T, max_q, max_kv, heads, kv heads, head_dim

    def call(n):
        R, T, max_q, max_kv, heads, H, D = args
        return L.moin_kv_attention(_kv(lib, heads=H), _tables(lib, n_rows=R), None, A, A, R, T, max_q, max_kv, A, heads * D, heads, 0.125, None, 0,
                                   A, heads * D, A, n, None)

    sizes = {}
    for v in (AUTO, ROWS, TENSOR):
        option(v)
        sizes[v] = L.moin_kv_attention_workspace_bytes(*args)
        assert call(sizes[v]) == NO_DEVICE and call(sizes[v] - 1) == WORKSPACE
    assert sizes[ROWS] < sizes[TENSOR]
    option(TENSOR)
    assert call(sizes[ROWS]) == WORKSPACE
    option(ROWS)
    assert call(sizes[TENSOR]) == NO_DEVICE
