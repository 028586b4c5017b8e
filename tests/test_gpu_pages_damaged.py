"""Page calls on a cache that is damaged: entries that a call cannot use are reported and left as they are, and the
call's other entries are carried out.  Every table entry, length, count of holders and stored value equals the
oracle's (the counts' own rule, one for each holder, does not hold for a damaged sequence)."""
import pytest
import torch

from tests.gpu_common import lsp_lib
from tests.target_common import make_cache, make_pool, same_cache, up
from tests.test_gpu_pages import Both, gen

pytestmark = pytest.mark.gpu
WIDTH, PAGE = 6, 16


@pytest.fixture(scope="module")
def lsp():
    return lsp_lib()


class Damaged(Both):
    def check(self):
        torch.cuda.synchronize()
        same_cache(self.o, self.k, self.v, *self.t)

    def set_len(self, s, n):
        self.t[1][s] = n
        self.o.len[s] = n

    def set_page(self, s, col, pg):
        self.t[0][s, col] = pg
        self.o.table[s, col] = pg

    def write_rows(self, seqs, start, g, bits):
        kn, vn = (torch.randn(start[-1], self.c.nkv, self.c.d, generator=g).to(self.k.dtype).cuda() for _ in range(2))
        self.lsp.lsp_pages_write(self.c, 0, self.ints(seqs), self.ints(start), kn, vn, self.err)
        self.o.write(0, seqs, start, up(kn), up(vn))
        assert self.bits() == bits


def damaged(lsp, lens, pages=24, dtype="bf16"):
    pool = make_pool(2, pages, 2, PAGE, 64, dtype, gen(3), device="cuda")
    table, lens, refs = make_cache(lens, 0, PAGE, pool, spare=0)
    wide = torch.full((table.shape[0], WIDTH), -1, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    return Damaged(lsp, pool, wide, lens, refs)


# below 0, one token more than the row of the table holds, and the ends of the type
LENGTHS = [-1, -3, WIDTH * PAGE + 1, 2 ** 31 - 1, -2 ** 31]


@pytest.mark.parametrize("n", LENGTHS)
def test_fork_leaves_sequences_of_no_length(lsp, n):
    b = damaged(lsp, [30, 40, 20, 0, 50])
    b.set_len(1, n)
    b.fork([1, 0], [3, 2])                           # the first source is damaged, the second pair is in order
    b.check()
    b.fork([4, 0], [1, 3])                           # a damaged destination
    b.check()


@pytest.mark.parametrize("n", LENGTHS)
def test_trim_and_reserve_leave_sequences_of_no_length(lsp, n):
    b = damaged(lsp, [30, 40, 20, 0])
    b.set_len(1, n)
    b.trim([1, 0], [5, 5])
    b.check()
    b.trim([1], [0])
    b.check()
    bad, short = b.reserve([1, 3, 0], [20, 20, 20])
    assert bad == [0] and not short
    b.check()
    b.reserve([1], [0])
    b.check()
    b.reserve([0, 1, 2], [7, 1, 50])
    b.check()


@pytest.mark.parametrize("n", LENGTHS)
def test_write_leaves_sequences_of_no_length(lsp, n):
    b = damaged(lsp, [30, 96, 20])
    b.set_len(1, n)
    b.write_rows([0, 1, 2], [0, 3, 8, 12], gen(1), lsp.LSP_DEV_BAD_SEQ)
    b.check()
    b.write_rows([0, 2], [0, 3, 12], gen(2), 0)
    b.check()


def test_the_longest_length_that_fits_is_in_order(lsp):
    b = damaged(lsp, [30, WIDTH * PAGE, 0])
    b.write_rows([1], [0, 20], gen(1), 0)
    b.fork([1], [2])
    assert b.reserve([2], [1]) == ([0], [])
    b.trim([1], [WIDTH * PAGE - 1])
    b.reserve([1], [1])
    b.check()
    assert int(b.t[1][1]) == WIDTH * PAGE


STRAYS = [-1, -7, 24, 10 ** 6, -2 ** 31]             # the pool has 24 pages


@pytest.mark.parametrize("pg", STRAYS)
def test_fork_and_trim_leave_sequences_with_a_page_of_no_pool(lsp, pg):
    b = damaged(lsp, [50, 40, 20, 33, 0])
    b.set_page(0, 1, pg)
    b.fork([0, 1], [4, 2])                           # a damaged source, and a pair in order
    b.check()
    b.fork([1, 3], [0, 4])                           # a damaged destination
    b.check()
    b.trim([0, 1], [3, 3])                           # it would let go of the stray page
    b.check()
    b.trim([0], [32])                                # only of a later one
    b.check()
    b.trim([0], [0])
    b.check()


@pytest.mark.parametrize("pg", STRAYS)
def test_reserve_and_write_leave_a_last_page_of_no_pool(lsp, pg):
    b = damaged(lsp, [50, 40, 20])
    b.set_page(1, 2, pg)                             # tokens 32 to 39
    bad, _ = b.reserve([0, 1, 2], [1, 1, 30])
    assert bad == [1]
    b.check()
    b.write_rows([0, 1, 2], [0, 1, 13, 15], gen(4), lsp.LSP_DEV_BAD_SEQ)     # rows of tokens 28 to 39: the first four have a place
    b.check()


def test_many_columns(lsp):
    """A sequence of more pages than a block has threads, the stray one among the last."""
    pool = make_pool(1, 700, 1, PAGE, 64, "bf16", gen(3), device="cuda")
    b = Damaged(lsp, pool, *make_cache([600 * PAGE, 20, 0], 0, PAGE, pool, spare=0))
    keep = b.t[0][0, 590].item()
    b.set_page(0, 590, 700)
    b.fork([0, 1], [2, 0])
    b.check()
    b.trim([0], [400 * PAGE])
    b.check()
    b.set_page(0, 590, keep)
    b.fork([0], [2])
    b.trim([0], [100 * PAGE - 3])
    b.check()


@pytest.mark.parametrize("fill", [0, 0xAB, 0xFF])
def test_compaction_leaves_entries_that_name_free_pages(lsp, fill):
    """Whatever the workspace holds: free pages at, past and before the live count, and pages of no pool."""
    b = damaged(lsp, [50, 40, 20, 33], pages=40)
    live = int((b.t[2] > 0).sum())
    free = [pg for pg in range(40) if int(b.t[2][pg]) == 0]
    assert any(pg >= live for pg in free) and any(pg < live for pg in free)
    b.set_page(0, 1, free[-1])
    b.set_page(1, 0, next(pg for pg in free if pg >= live))
    b.set_page(1, 2, next(pg for pg in free if pg < live))
    b.set_page(2, 0, 40)
    b.set_page(3, 2, -5)
    b.ws.fill_(fill)
    b.compact()
    b.check()


@pytest.mark.parametrize("n", LENGTHS)
def test_compaction_keeps_the_pages_of_a_sequence_of_no_length(lsp, n):
    """Its pages are moved like the others; its table follows, so that a length that is put right finds them."""
    b = damaged(lsp, [50, 40, 20, 33], pages=40)
    want = [[x.copy() for x in b.o.tokens(layer, 1)] for layer in range(2)]
    b.set_len(1, n)
    b.compact()
    b.check()
    b.set_len(1, 40)
    for layer in range(2):
        for pool, x in zip((b.k, b.v), want[layer]):
            got = up(pool[layer, b.t[0][1, :3].long()].transpose(1, 2).flatten(0, 1)[:40])
            assert (got == x).all()
