"""NaN in attention: a row is NaN exactly where its formula is, and nothing else changes.

A key with a NaN makes the output and lse of every row that sees it NaN, so does a NaN in the row's own query; a value
with a NaN makes those dims NaN of every row that sees it, whatever its weight.  Rows that do not see it yet are as
without it: they are compared with the fp64 oracle within the tolerances of test_gpu_prefix_attn.py.
"""
import numpy as np
import pytest
import torch

from oracle.target import PagedCache, cache_attention
from tests import target_common
from tests.gpu_common import lsp_lib
from tests.q4_common import held
from tests.target_common import DT, up
from tests import test_gpu_prefix_attn as wide, test_gpu_prefix_attn_q4 as packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


def scales(pool):
    """[layers][pages][nkv][page][d / 32] of a pool of bytes, as 16-bit words that may be written."""
    page, width = pool.shape[3:]
    d = width * 16 // 9
    return pool.flatten(3)[..., page * d // 2:].view(torch.int16).unflatten(-1, (page, d // 32))


def spoil(pool, table, seq, tokens, head, group, word=0x7FC0):
    x, page = scales(pool), pool.shape[3]
    for t in tokens:
        x[0, int(table[seq, t // page]), head, t % page, group] = word


def check(k, v, t, q, rows, out, z, seen=True):
    """seen=False: rows that see a NaN or infinite value are left out."""
    table, lens, refs = (x.cpu().numpy() for x in t)
    nq, d, rep = q.shape[1], q.shape[2], q.shape[1] // k.shape[2]
    oc = PagedCache(np.where(np.isfinite(k), k, 0), np.where(np.isfinite(v), v, 0), table, lens, refs)
    whole = PagedCache(k, v, table, lens, refs)
    start = np.concatenate([[0], np.cumsum(rows)]).astype(int)
    qf = up(q)
    want, lse, size = cache_attention(oc, 0, np.where(np.isfinite(qf), qf, 0), list(range(len(rows))), start, d ** -0.5)
    lost, lost_z = np.zeros(want.shape, bool), np.zeros(lse.shape, bool)
    for i, r in enumerate(rows):
        kk, vv = (~np.isfinite(x) for x in whole.tokens(0, i))
        for j in range(r):
            n = int(lens[i]) - r + j + 1
            for h in range(nq):
                lost_z[start[i] + j, h] = kk[:n, h // rep].any() or np.isnan(qf[start[i] + j, h]).any()
                lost[start[i] + j, h] = vv[:n, h // rep].any(0) | lost_z[start[i] + j, h]
    got, zg = out.double().cpu().numpy(), z.double().cpu().numpy()
    if seen:
        assert lost.any() and not lost.all()
        assert np.array_equal(np.isnan(got), lost)
        assert np.array_equal(np.isnan(zg), lost_z)
    tol = ((2 ** -8 + 2 ** -10) * (size + np.abs(want)) if q.dtype == torch.bfloat16 else 4e-5 * size) + 1e-30
    assert (np.abs(got - want)[~lost] <= tol[~lost]).all(), np.nanmax((np.abs(got - want) / tol)[~lost])
    assert (np.abs(zg - lse)[~lost_z] <= 2e-5 + 2e-6 * np.abs(lse[~lost_z])).all()


# rows of an item for both kernels of rows in bf16; of that on the tensor cores, one row tile and two
ROWS = {"few": ([1, 3], 4, 2), "one tile": ([20, 30], 4, 2), "two tiles": ([150, 90], 4, 2), "64 heads": ([1, 3], 64, 1)}


def made(name, dtype, d, own=0, seed=0):
    rows, nq, nkv = ROWS[name]
    lens = [512 + r + own for r in rows]
    pool, t, q = packed.case(lens, rows, 512, nq=nq, nkv=nkv, d=d, dtype=dtype, page=64, seed=seed)
    return pool, t, q, lens, rows


def both(lsp, pool, t, q, rows, seen=True):
    for shared in (512, 0):
        out, z = packed.attend(lsp, pool, t, q, list(range(len(rows))), rows, shared)
        check(*(held(x) for x in pool), t, q, rows, out, z, seen)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(ROWS))
def test_keys(lsp, name, d, dtype):
    # an own token's, alone behind the prompt; or the last row's
    for seq in (0, 1):
        pool, t, q, lens, rows = made(name, dtype, d)
        spoil(pool[0], t[0], seq, [lens[seq] - 1], 0, d // 32 - 1)
        both(lsp, pool, t, q, rows)
    # 16 tokens of the prompt, which one warp has; whole blocks of it
    for tokens in (range(16, 32), range(0, 128), range(256, 384)):
        if ROWS[name][2] == 1:                       # (one key head: no row would be left)
            break
        pool, t, q, lens, rows = made(name, dtype, d, own=70)
        spoil(pool[0], t[0], 0, tokens, 0, 0)
        both(lsp, pool, t, q, rows)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(ROWS))
def test_a_whole_sequence_of_keys(lsp, name, dtype):
    pool, t, q, lens, rows = made(name, dtype, 128, own=200)
    for group in range(4):
        spoil(pool[0], t[0], 1, range(512, lens[1]), 0, group)
    both(lsp, pool, t, q, rows)
    lens, rows = [40 + r for r in rows], rows        # nothing else to see
    pool, t, q = packed.case(lens, rows, 0, nq=q.shape[1], nkv=pool[0].shape[2], d=128, dtype=dtype, page=64)
    spoil(pool[0], t[0], 0, range(lens[0]), 0, 2)
    out, z = packed.attend(lsp, pool, t, q, [0, 1], rows, 0)
    check(*(held(x) for x in pool), t, q, rows, out, z)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(ROWS))
def test_queries(lsp, name, d, dtype):
    pool, t, q, lens, rows = made(name, dtype, d, own=30)
    q[0, 1, 5] = float("nan")
    q[-1, 0] = float("nan")
    both(lsp, pool, t, q, rows)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("name", list(ROWS))
def test_values(lsp, name, d, dtype):
    # of the prompt; of new tokens, which the rows before them do not see; of the token of the first row
    for seq, back, group in ((0, None, 0), (1, 1, d // 32 - 1), (1, 2, 0), (0, 1, 1), (1, 3, 1)):
        pool, t, q, lens, rows = made(name, dtype, d, own=9)
        tokens = [77, 300] if back is None else [lens[seq] - back]
        spoil(pool[1], t[0], seq, tokens, 0, group)
        both(lsp, pool, t, q, rows)
    # several groups and tokens of one call, and weights so small that fp32 has none of them
    pool, t, q, lens, rows = made(name, dtype, d, own=9)
    spoil(pool[1], t[0], 1, [lens[1] - 1], 0, 0)
    spoil(pool[1], t[0], 1, [lens[1] - 3, lens[1] - 2], 0, 1)
    both(lsp, pool, t, q, rows)
    out, z = packed.attend(lsp, pool, t, q * 200, [0, 1], rows, 512)
    k, v = (held(x) for x in pool)
    assert np.array_equal(np.isnan(up(out)), np.isnan(up(packed.attend(lsp, pool, t, q, [0, 1], rows, 512)[0])))
    assert not z.isnan().any()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(ROWS))
def test_values_past_the_largest_bf16_number_stay_out_of_rows_that_do_not_see_them(lsp, name, dtype):
    pool, t, q, lens, rows = made(name, dtype, 128, own=9)
    at = lens[1] - 1
    spoil(pool[1], t[0], 1, [at], 0, 1, word=0x7E18)             # 1.1875 x 2^125: 7 of it are past 2^128
    page = 64
    block = pool[1][0, int(t[0][1, at // page]), 0].flatten()
    block[(at % page) * 64:(at % page) * 64 + 64] = 0xFF         # codes 7
    both(lsp, pool, t, q, rows, seen=False)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("dtype", list(DT))
def test_many_sequences_with_a_nan_here_and_there(lsp, dtype, seed):
    """Short segments one behind the other, each with its own."""
    rng = np.random.RandomState(seed)
    n = 90
    rows = [int(x) for x in rng.randint(1, 6, n)]
    lens = [r + int(x) for r, x in zip(rows, rng.randint(0, 300, n))]
    nq, nkv, d = (64, 1, 64) if seed % 2 else (40, 2, 128)
    pool, t, q = packed.case(lens, rows, 0, nq=nq, nkv=nkv, d=d, dtype=dtype, page=32, seed=seed)
    for i in rng.permutation(n)[:40]:
        spoil(pool[int(rng.randint(2))], t[0], int(i), [int(rng.randint(lens[i]))], 0, int(rng.randint(d // 32)))
    out, z = packed.attend(lsp, pool, t, q, list(range(n)), rows, 0)
    check(*(held(x) for x in pool), t, q, rows, out, z)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("name", list(ROWS))
def test_queries_and_keys_of_a_cache_that_holds_elements(lsp, name, dtype):
    rows, nq, nkv = ROWS[name]
    lens = [512 + r for r in rows]
    pool, t, q = wide.case(lens, rows, 512, nq=nq, nkv=nkv, d=128, dtype=dtype, page=64)
    q[0, 1, 5] = float("nan")
    pool[0][0, int(t[0][1, 8]), 0, 0, 3] = float("nan")          # the first own token's key
    for shared in (512, 0):
        out, z = wide.attend(lsp, pool, t, q, [0, 1], rows, shared)
        check(*(up(x) for x in pool), t, q, rows, out, z)
