"""GPU parity of keeping drafted tokens in rows that share pages: against the oracle, and with the tokens that a program appends next."""
import numpy as np
import pytest
import torch

import paper_2609_24270_amd as asym
from oracle import drafts, kv_pages
from tests.test_gpu_drafts import dev, i32  # noqa: F401

pytestmark = pytest.mark.gpu

PATHS = [[0], [0, 1], [], list(range(14)), list(range(45)), list(range(46)), [0, 1, 40], [0, 15, 16, 17]]


def shared(dev, H, seed):
    """Rows of 96 tokens, their last 46 drafted, each forked behind them (all pages shared), one without a fork."""
    R = len(PATHS) + 1
    g = torch.Generator().manual_seed(seed)
    total = 2 * R * H * 4 + 5
    pools = [torch.randn((total, 32, 128), generator=g).to(torch.bfloat16).to(dev) for _ in range(2)]
    table, lens, refs = torch.full((2 * R, H, 6), -1, dtype=torch.int32, device=dev), i32([0] * 2 * R, dev), i32([0] * total, dev)
    asym.kv_extend(table, lens, refs, i32(list(range(R)), dev), i32([96] * R, dev))
    asym.kv_fork(*pools, table, lens, refs, i32(list(range(R - 1)), dev), i32(list(range(R, 2 * R - 1)), dev))
    return R, pools, table, lens, refs


@pytest.mark.parametrize("H", [1, 3, 70])
def test_rows_do_not_end_inside_a_page_of_another(dev, H):
    R, pools, table, lens, refs = shared(dev, H, H)
    paths = PATHS + [[0]]
    path = sum([p + [-1] * (46 - len(p)) for p in paths], [])
    cu, count = [46 * i for i in range(R + 1)], [len(p) for p in paths]
    rows = list(range(R))
    words = [p.view(torch.int16).cpu().numpy() for p in pools]
    c = kv_pages.Cache(table.cpu().numpy(), lens.cpu().numpy(), refs.cpu().numpy(), words)
    forks = [p.clone() for p in pools]
    # (row by row: rows of one call share no drafted tokens here, but the oracle takes them one after the other)
    drafts.keep(c, rows, cu, path, count)
    asym.kv_keep(*pools, table, lens, refs, i32(rows, dev), i32(cu, dev), i32(path, dev), i32(count, dev))
    assert lens.tolist() == c.lens.tolist()
    assert c.lens[:R].tolist() == [96, 96, 96, 64, 96, 96, 96, 96, 51]
    for want, got in zip((*c.pools, c.table, c.refs), (*[p.view(torch.int16) for p in pools], table, refs)):
        assert np.array_equal(want, got.cpu().numpy())
    # the rows grow, and their forks stay as they are
    start = lens[:R].clone()
    asym.kv_extend(table, lens, refs, i32(rows, dev), start + 20)
    assert lens[:R].tolist() == (start + 20).tolist()
    new = torch.full((R * 20, H, 128), 7.0, dtype=torch.bfloat16, device=dev)
    tables = table[:R].contiguous()
    asym.kv_append(new, new, *pools, tables, tables, i32([20 * i for i in range(R + 1)], dev), start)
    for r in range(R, 2 * R - 1):
        pages = table[r, :, :3].long().flatten()
        assert all(torch.equal(p[pages], f[pages]) for p, f in zip(pools, forks))
