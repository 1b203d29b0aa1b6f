"""Drafted trees at the ends of what their inputs may hold: values that are not finite, groups and thresholds
at the end of fp16's range, full caches, and decode steps after an acceptance."""
import numpy as np
import pytest

from test_gpu_tree import Held, admitted, check, dev, drafts, workload

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_07966_amd import _lib
    _lib.lib()


def attend(c, q, kt, vt, mask, **kw):
    return c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64)), **kw).cpu().numpy()


def rest_right(wl, books, q, kt, vt, mask, got, clean, rows, channels=slice(None)):
    """`got` against the oracle with the finite kt and vt, but for some rows' channels.  (Not bit for bit `clean`:
    the rows of a wave move their softmax references together, so one row's logits decide about the roundings of
    another's probabilities.)"""
    out = got.copy()
    out[:, rows, :, channels] = clean[:, rows, :, channels]
    for s in range(wl.n_seqs):
        check(wl, Held(wl, books, s), s, q[s], kt[s], vt[s], mask[s], out[s], q.shape[1])


def only(s, n, seen):
    """Masks of all zeros but for rows {row: [nodes]}."""
    mask = np.zeros((s, n), np.uint64)
    for row, nodes in seen.items():
        mask[:, row] = sum(1 << j for j in nodes)
    return mask


# ---- values that are not finite -----------------------------------------------------------------------

@pytest.mark.parametrize("name", ["FP16", "UQ4-g64", "KVQ4"])
@pytest.mark.parametrize("hq,hkv,d,n", [(4, 4, 64, 8), (8, 2, 128, 8), (8, 4, 64, 32), (8, 1, 64, 64)])
@pytest.mark.parametrize("lens", [[512], [40], [512, 1100, 40]])
def test_a_nan_that_a_row_sees_is_shown(name, hq, hkv, d, n, lens):
    """A NaN in a node's key makes every row that attends to the node NaN and no other, however the cache is
    split: in a range of the drafted tokens alone, in one with cached tokens, and without splits."""
    wl = workload([name] * len(lens), lens, hq, hkv, d)
    rng = np.random.default_rng(31)
    c, books = admitted(wl, 4)
    q, kt, vt = drafts(wl, rng, n)
    mask = only(len(lens), n, {0: [0], 1: [0, 1], 2: [2], 3: [2, n - 1], 5: [0, 2, 5], n - 1: [n - 1]})
    clean = attend(c, q, kt, vt, mask)
    assert np.all(np.isfinite(clean))
    for node, rows in ((0, (0, 1, 5)), (2, (2, 3, 5)), (n - 1, (3, n - 1))):
        bad = kt.copy()
        bad[:, node, :, 7] = np.nan
        got = attend(c, q, bad, vt, mask)
        assert np.all(np.isnan(got[:, list(rows)])), node
        rest_right(wl, books, q, kt, vt, mask, got, clean, list(rows))
    # and a NaN in a query is its own row's
    bad = q.copy()
    bad[:, 4, :, 3] = np.nan
    got = attend(c, bad, kt, vt, mask)
    assert np.all(np.isnan(got[:, 4]))
    rest_right(wl, books, q, kt, vt, mask, got, clean, [4])
