"""GPU: operators over drafted token trees where calls go wrong beside calls that are right: rows and trees that are
refused next to good ones, tables and stacks with holes, committed K/V that are not finite or very large, and the same rows
joined along every path.  References and tolerances are those of test_gpu_tree.py."""
import numpy as np
import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import tree
from test_gpu_tree import (HEADS, HostPages, _attend, _batch, _cache, _close, _dev, _drafts, _host_rows, _mixed, _q, _say,
                           _shape, _upload, _want, _ws, random_parents)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rows that are skipped beside rows that are not

@pytest.mark.parametrize("field,value", [("seq", -1), ("c", 99)])
@pytest.mark.parametrize("hd,H,trees,n,good,max_nodes", [(128, 16, 16, 16, 8, 16), (64, 55, 4, 16, 2, 16),
                                                         (64, 20, 8, 32, 4, 32), (64, 55, 4, 64, 1, 64)])
def test_skipped_rows_take_nothing_from_the_others(hd, H, trees, n, good, max_nodes, field, value):
    """Contexts of several segments; all trees fill the chip, the good ones do not.  Bit for bit what the good rows get
    without the bad ones, and what 64-bit arithmetic gets."""
    shape = _shape(hd, H)
    rng = np.random.default_rng(trees)
    made = [(1024 + 37 * (t // (trees // good)), random_parents(rng, n)) for t in range(trees)]
    at = [t // (trees // good) for t in range(trees)]  # the good trees' sequences; the others share their neighbour's
    b = _batch(rng, made, [1] * trees)
    ok = b.seq % (trees // good) == 0
    b.seq = np.array([at[t] for t in b.seq], np.int32)
    getattr(b, field)[~ok] = value
    kv, pt = _cache(shape, [(1, made[t][0] + n) for t in range(0, trees, trees // good)], 3)
    q = _q(shape, b.n, 7)
    keep = np.flatnonzero(ok)
    sel = torch.from_numpy(keep).cuda()
    _say(f"[gpu] tree attention {H} x {hd}: {good} of {trees} trees of {n} are good ({field} {value})")
    alone = _attend(shape, kv, b.take(keep), q[sel].contiguous(), max_nodes)[:len(keep)]
    got = _attend(shape, kv, b, q, max_nodes, fill=3.0, check=cdb.CDB_DEV_UNMAPPED_PAGE)[:b.n]
    assert bool((got[torch.from_numpy(~ok).cuda()] == 3.0).all())
    assert torch.equal(got[sel], alone)
    some = keep[:: max(1, len(keep) // 6)]
    want, tol = _want(shape, kv, pt, b.take(some), q[torch.from_numpy(some).cuda()])
    _close(got[torch.from_numpy(some).cuda()], want, tol)
