"""What the attention entry points promise of workspace sizes, and how many positions a table may have: nothing here touches a device."""
import ctypes as C
import random

import pytest

from paper_2602_11688_amd import attention as ga

FAKE = 4096                                              # an aligned address that no call here looks at


def _bytes(S, T, columns, *, q_heads=32, kv_heads=8, d=128, page=512, type=0, token=False):
    scales = FAKE if type == 2 else None
    cache = ga._Cache(FAKE, FAKE, scales, scales, type, 10, page, kv_heads, d, 0, kv_heads * page * d, page * d, d)
    batch = ga._Batch(S, T, columns, 0, FAKE, FAKE, None if token else FAKE)
    n = C.c_size_t()
    assert ga._lib().gorgo_attend_workspace_bytes(C.byref(cache), C.byref(batch), q_heads, C.byref(n)) == 0, ga._lib().gorgo_last_error()
    return n.value


@pytest.mark.parametrize("how", [dict(), dict(q_heads=4, kv_heads=1, d=64, page=64), dict(d=80, page=48, type=2), dict(q_heads=71, kv_heads=1),
                                 dict(q_heads=16, kv_heads=16, d=64, type=1), dict(q_heads=1024, kv_heads=256)])
def test_a_workspace_of_a_large_batch_fits_every_smaller_one(how):
    """Fewer sequences, fewer tokens, fewer columns, prompts or single tokens: few rows are split where many are not, and need no more."""
    rng = random.Random(7)

    def some(most):
        return max(1, int(most ** rng.random()))
    for _ in range(300):
        S = some(64)
        T, columns = max(S, some(60000)), some(4000)
        large = _bytes(S, T, columns, **how)
        for _ in range(20):
            s = some(S)
            assert _bytes(s, max(s, some(T)), some(columns), **how) <= large
            assert _bytes(s, s, some(columns), token=True, **how) <= large


def test_workspaces_stay_small():
    """Whatever the batch: at most a row of 128 values and two numbers of each row that all compute units hold at once, or of single tokens'
    partial rows, and the counts."""
    for S, T in ((1, 1), (8, 500), (8, 20000), (1, 2 ** 20), (64, 64)):
        for how in (dict(), dict(q_heads=32, kv_heads=1), dict(d=64), dict(q_heads=71, kv_heads=1)):
            assert 2048 <= _bytes(S, T, 4000, **how) <= 2048 + 512 * 256 * (64 + 2) * 4 + 256


@pytest.mark.parametrize("columns,page,ok", [(65538, 32767, False), (2 ** 31 - 1, 1, False), (2 ** 31 - 1023, 1, False), (2 ** 31 - 1024, 1, True), (2 ** 21 - 1, 1024, True),
                                             (2 ** 21, 1023, True), (2 ** 21, 1024, False)])
def test_tables_of_nearly_32_bits_of_positions(columns, page, ok):
    """The kernels' positions go up to two steps of keys beyond the last, and have to stay below 2^31 there."""
    cache = ga._Cache(FAKE, FAKE, None, None, 0, 10, page, 2, 64, 0, 2 * page * 64, page * 64, 64)
    batch = ga._Batch(3, 3, columns, 0, FAKE, FAKE, None)
    n = C.c_size_t()
    L = ga._lib()
    assert L.gorgo_attend_workspace_bytes(C.byref(cache), C.byref(batch), 8, C.byref(n)) == (0 if ok else -1)
    if not ok:                                           # (a call that is accepted would look at the addresses)
        assert b"table_columns" in L.gorgo_last_error()
        rows, how = ga._Rows(FAKE, 8 * 64, 64), ga._Attention(8, 0, 0.125, 0)
        for f in (L.gorgo_attend_prompt, L.gorgo_attend_token):
            assert f(C.byref(cache), C.byref(batch), C.byref(how), C.byref(rows), C.byref(rows), None, FAKE, 1 << 40, None) == -1
        for f in (L.gorgo_kv_write, L.gorgo_kv_read):
            assert f(C.byref(cache), C.byref(batch), C.byref(rows), C.byref(rows), None) == -1


def test_scales_that_overflow_in_powers_of_two_are_refused():
    """The kernels multiply by scale * log2(e): a scale near the end of 32 bits makes that infinite, and a score of 0 NaN."""
    cache = ga._Cache(FAKE, FAKE, None, None, 0, 10, 16, 2, 64, 0, 2 * 16 * 64, 16 * 64, 64)
    batch, rows = ga._Batch(3, 3, 400, 0, FAKE, FAKE, None), ga._Rows(FAKE, 8 * 64, 64)
    for scale, code in ((3.0e38, -6), (2.3e38, -7)):     # (no workspace: the one that is taken is refused for that)
        how = ga._Attention(8, 0, scale, 0)
        assert ga._lib().gorgo_attend_token(C.byref(cache), C.byref(batch), C.byref(how), C.byref(rows), C.byref(rows), None, None, 0, None) == code
