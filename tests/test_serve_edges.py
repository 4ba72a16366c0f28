"""The operators around a verification at the ends of what their documentation allows: wide tables, extreme scores, places far
into a cache, large trees and many of them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_serve_ops import BF, HF, Attn, binding, drafts, handle, tree  # noqa: E402,F401


@pytest.mark.parametrize("G,d,width", [(64, 128, 2 ** 21 + 5), (8, 128, 2 ** 21 + 5), (64, 128, 2 ** 24 + 5)])
def test_commit_of_wide_tables(binding, G, d, width):
    """Every slot of the table is a good one; only what the counts leave is copied, from the first position to the last."""
    L, B, R, pages, page = 1, 2, 4, 5, 8
    pool = [torch.randn((L, pages, page, G, d)).to(BF).cuda() for _ in range(2)]
    k, v = (torch.randn((L, B, R, G, d)).to(BF).cuda() for _ in range(2))
    slots = torch.full((B, width), 3, dtype=torch.int64, device="cuda")
    row = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    h = handle(binding, B, tree(1))
    cache = binding.PagedCache(*pool)
    for counts, at in (([0, -1], []), ([-2 ** 31, 0], []), ([2, width], [(0, 0, 2, 9), (0, 1, 0, 39), (1, 0, 3, 17), (1, width - 1, 1, 30), (1, width // 2, 0, 1)]),
                       ([1, width - 1], [(0, 0, 1, 4), (1, width - 2, 2, 12)]), ([2 ** 31 - 1, 0], [(0, width - 1, 3, 0)])):
        want = [x.clone() for x in pool]
        row.fill_(-1)
        if not at:
            row.fill_(0)                                  # all of them good rows as well
        for b, j, r, s in at:
            row[b, j], slots[b, j] = r, s
            want[0][:, s // page, s % page], want[1][:, s // page, s % page] = k[:, b, r], v[:, b, r]
        if at:                                            # behind the counts: rows that may not be copied
            for b in range(B):
                row[b, max(0, min(counts[b], width)):] = 0
        h.cache_commit(cache, k, v, slots, row, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(pool[0], want[0]) and torch.equal(pool[1], want[1]), counts
        for b, j, r, s in at:
            slots[b, j] = 3
