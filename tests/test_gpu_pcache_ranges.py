"""The paged token cache at the ends of its ranges: tables that were written by hand."""
import pytest
import torch

from oracle import pcache as op
from tests.test_gpu_pcache import as_lists, ctx, fc, moved, plain, pool, run_step  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------ pages
def compact(fc, ctx, caches):  # noqa: F811
    """A compaction against the oracle; entries that are no page stay as they are."""
    state, R = caches[0].pages, caches[0].k.shape[2]
    pages, table = op.Pages(as_lists(state), state.n_pages, R, state.max_pages), state.table.tolist()
    before = [plain(c) for c in caches]
    live = torch.full((1,), -5, dtype=torch.int32, device="cuda")
    fc.fc_pcache_compact(ctx, caches, live)
    torch.cuda.synchronize()
    L, moves = pages.compact()
    assert live.item() == L
    assert state.table.tolist() == [[x if p is None else p for p, x in zip(*rows)] for rows in zip(pages.table, table)]
    assert state.holders.tolist() == pages.holders()
    for c, (k, v) in zip(caches, before):
        k2, v2 = plain(c)
        assert torch.equal(k2, moved(k, moves, R)) and torch.equal(v2, moved(v, moves, R)), "rows moved"
    return len(moves)


@pytest.mark.parametrize("B,M,P", [(3, 5, 40), (2, 4, 7200)])
def test_compaction_of_a_table_written_by_hand(fc, ctx, B, M, P):  # noqa: F811
    """Entries that no step has counted are held all the same, whatever the holders' counts say: a page that the
    table names is not written over, and one that it does not name is free.  A pool whose counts a
    workgroup holds in LDS, and a larger one."""
    g = torch.Generator().manual_seed(P)
    R, kv, hd = 16, 1, 64
    state = fc.PageState.alloc(B, M, P)
    caches = [pool(g, state, kv, hd, R, fc) for _ in range(2)]
    run_step(fc, ctx, caches, None, [0] * B, [R * 3] * B, R * 3)
    # pages named by hand, some of them twice, and entries that are no page
    state.table[0, 0], state.table[0, 3], state.table[1, 3], state.table[1, 0] = P - 1, P - 3, P - 3, P
    state.table[B - 1, 1] = -9
    assert compact(fc, ctx, caches) > 0
    state.holders.copy_(torch.arange(P, dtype=torch.int32, device="cuda") % 3 - 1)
    state.table[0, 1] = P // 2
    assert compact(fc, ctx, caches) == 1
    state.table.fill_(-1)
    assert compact(fc, ctx, caches) == 0
