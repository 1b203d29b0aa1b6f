"""Drafted trees at the ends of what their inputs may hold: values that are not finite, groups and thresholds
at the end of fp16's range, full caches, and decode steps after an acceptance."""
import numpy as np
import pytest

from test_gpu_tree import CONFIGS, Held, U, admitted, check, dev, drafts, exports, same_state, trees, workload
from workloads import step_inputs

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


# ---- the end of fp16's range -----------------------------------------------------------------------------

def bounded(keys, vals, ekey, evals, q, kt, vt, mask, out):
    """One sequence: keys, vals [Hkv] of [n][d] and bounds e_k, e_v of their errors alike; q, out [N][Hq][d].

    With u = 2^-11 (half an fp16 step relative to the value) an output is off by at most u |o| (its rounding)
    + u sum p |v| (probabilities) + sum p e_v (values) + (exp(2 dl) - 1) sum p |v| (keys: a logit is off by at
    most dl = sum |q| e_k / sqrt(d)) + 1e-5 sum p |v| (sums and exponentials in float32)."""
    n, hq, d = q.shape
    g = hq // len(keys)
    for h in range(len(keys)):
        for i in range(n):
            seen = [j for j in range(n) if int(mask[i]) >> j & 1]
            none = np.zeros((len(seen), d))
            k, v = (np.vstack([x, y[seen, h].astype(np.float64)]) for x, y in ((keys[h], kt), (vals[h], vt)))
            ek, ev = np.vstack([ekey[h], none]), np.vstack([evals[h], none])
            qq = q[i, h * g:(h + 1) * g].astype(np.float64)
            z = qq @ k.T / np.sqrt(d)
            p = np.exp(z - z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            ref, mag = p @ v, p @ np.abs(v)
            dl = (np.abs(qq) @ ek.T).max(1, keepdims=True) / np.sqrt(d)
            tol = U * np.abs(ref) + p @ ev + (U + np.expm1(2 * dl) + 1e-5) * mag
            err = np.abs(out[i, h * g:(h + 1) * g].astype(np.float64) - ref)
            assert np.all(err <= tol), (h, i, float(np.nanmax(err / tol)), bool(np.isfinite(out).all()))


def uq_error(x, eff):
    """x [...][64] groups, eff what their codes stand for: the value's own rounding, u |v|, and those of the
    group's middle and step, a whole unit of each where the range ends at fp16's: 2 u (|mid| + |v - mid|)."""
    mn, mx = (f(x.astype(np.float64), axis=-1, keepdims=True) for f in (np.min, np.max))
    mid = mn + 8 * (mx - mn) / 15
    return U * np.abs(eff) + 2 * U * (np.abs(mid) + np.abs(eff - mid)) + 2.0 ** -21


def ranged(rng, shape, ends):
    """Groups of 64 along the last axis, each between a pair of ends and touching both."""
    x = np.empty(shape, np.float64)
    pick = np.array(ends, np.float64)[rng.integers(0, len(ends), shape[:-1])]
    x[:] = pick[..., :1] + (pick[..., 1:] - pick[..., :1]) * rng.random(shape)
    x[..., 0], x[..., 63] = pick[..., 0], pick[..., 1]
    return rng.permuted(x, axis=-1).astype(np.float16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("what", ["values", "keys"])
def test_uniform_groups_at_the_end_of_fp16(d, what):
    """Groups whose least or greatest value is the last finite one, or near it."""
    from oracle import uniform
    from paper_2609_07966_amd.cache import KVCache
    rng = np.random.default_rng(34)
    lens, hq, hkv, n = [64, 150, 700], 4, 2, 6
    t = sum(lens)
    m = 65504.0
    ends = [(0, m), (-m, m), (-m, 0), (m - 64, m), (-m, -60000), (m, m)] + [(float(x), m) for x in rng.integers(-m, m, 40)] + \
        [(-m, float(x)) for x in rng.integers(-m, m, 40)] + [(float(x), 64064.0) for x in rng.integers(-m, 64000, 20)]
    k, v = (rng.standard_normal((t, hkv, d)).astype(np.float16) for _ in range(2))
    if what == "values":
        v = ranged(rng, (t, hkv, d // 64, 64), ends).reshape(t, hkv, d)
    else:  # channels 0 to 7 of every whole block
        row = 0
        for n0 in lens:
            whole = n0 // 64 * 64
            x = ranged(rng, (whole // 64, hkv, 8, 64), ends)  # [block][head][channel][token]
            k[row:row + whole, :, :8] = x.transpose(0, 3, 1, 2).reshape(whole, hkv, 8)
            row += n0
    c = KVCache((3, hq, hkv, d, 4), [{"method": "uq", "bits": 4, "group": 64}] * 3, lens)
    c.append_prompt(dev(k), dev(v))
    q, kt, vt = (rng.standard_normal((3, n, h, d)).astype(np.float16) for h in (hq, hkv, hkv))
    if what == "keys":  # logits of a few units, most of their terms from the large channels
        q[..., :8] = (rng.standard_normal((3, n, hq, 8)) * 2.0 ** -13).astype(np.float16)
    mask, _ = trees(rng, 3, n)
    mask[:, 0] = 0
    got = attend(c, q, kt, vt, mask)
    row = 0
    for s, n0 in enumerate(lens):
        parts = [[], [], [], []]
        for h in range(hkv):
            kh, vh, whole = k[row:row + n0, h], v[row:row + n0, h], n0 // 64 * 64
            ke, ve = uniform.effective_keys(kh, 4, 64), uniform.effective_values(vh, 4, 64)
            ek, groups = np.zeros((n0, d)), lambda x: x.reshape(-1, 64, d).transpose(0, 2, 1)
            ek[:whole] = uq_error(groups(kh[:whole]), groups(ke[:whole])).transpose(0, 2, 1).reshape(whole, d)
            ev = uq_error(vh.reshape(n0, -1, 64), ve.reshape(n0, -1, 64)).reshape(n0, d)
            for part, x in zip(parts, (ke, ve, ek, ev)):
                part.append(x)
        bounded(*parts, q[s], kt[s], vt[s], mask[s], got[s])
        row += n0


@pytest.mark.parametrize("name", ["FP16", "UQ4-g64", "KVQ3"])
@pytest.mark.parametrize("lens", [[63, 129], [900, 2100]])
def test_rows_beside_a_node_that_is_not_finite(name, lens):
    """Rows that attend to several nodes but not to the one whose key and value are not finite: against the
    oracle with the whole of their masks."""
    wl = workload([name] * 2, lens, 8, 2, 128)
    rng = np.random.default_rng(33)
    c, books = admitted(wl, 4)
    n = 12
    q, kt, vt = drafts(wl, rng, n)
    mask, _ = trees(rng, 2, n)
    mask &= ~np.uint64(1 << 3)
    mask[:, 3] |= np.uint64(1 << 3)
    mask[:, 11] |= np.uint64(0x7F7)
    clean = attend(c, q, kt, vt, mask)
    for bad in (np.nan, np.inf, -np.inf):
        kb, vb = kt.copy(), vt.copy()
        vb[:, 3] = bad
        kb[:, 3, :, ::2] = bad
        got = attend(c, q, kb, vb, mask)
        assert not np.any(np.isfinite(got[:, 3]))
        rest_right(wl, books, q, kt, vt, mask, got, clean, [3])


@pytest.mark.parametrize("name", ["FP16", "KVQ3"])
@pytest.mark.parametrize("hq,hkv,d,n", [(4, 4, 64, 13), (4, 4, 128, 40), (8, 4, 64, 24), (4, 4, 64, 64), (8, 2, 128, 50)])
@pytest.mark.parametrize("lens", [[40], [70], [300] * 64, [1500]])
def test_an_infinite_value_that_a_row_sees_stays_infinite(name, hq, hkv, d, n, lens):
    """A node's infinite value has a positive weight in the rows that attend to it, whichever of the others
    they see: the output is infinite there and what it was anywhere else."""
    wl = workload([name] * len(lens), lens, hq, hkv, d)
    rng = np.random.default_rng(32)
    c, books = admitted(wl, 4)
    q, kt, vt = drafts(wl, rng, n)
    mask, _ = trees(rng, 1, n)
    mask = np.tile(mask, (len(lens), 1))
    mask[:, n - 1] = np.uint64(1 << (n - 1))  # a row that sees the last node alone
    mask[:, n - 2] = np.uint64(3 << (n - 2))
    clean = attend(c, q, kt, vt, mask)
    for node, bad in ((n - 1, np.inf), (n - 2, -np.inf), (0, np.inf)):
        odd = vt.copy()
        odd[:, node, :, 5:9] = bad
        got = attend(c, q, kt, odd, mask)
        sees = [i for i in range(n) if int(mask[0, i]) >> node & 1]
        assert np.all(got[:, sees][..., 5:9] == bad), node
        if len(lens) == 1:
            rest_right(wl, books, q, kt, vt, mask, got, clean, sees, slice(5, 9))


@pytest.mark.parametrize("name", ["FP16", "UQ4-g64", "KVQ4"])
@pytest.mark.parametrize("n0", [1, 5, 70, 700])
def test_a_mean_of_last_finite_values_is_finite(name, n0):
    """Every value of a channel is fp16's last finite one (or its negative): so is every weighted mean of
    them, whichever way the weights were rounded."""
    from paper_2609_07966_amd.cache import KVCache
    rng = np.random.default_rng(35)
    hq, hkv, d, n = 8, 2, 64, 64
    wl = workload([name], [n0], hq, hkv, d)
    books = np.concatenate([np.linspace(-1, 1, 1 << b) for b in (2, 3, 4) for _ in range(2)])
    c = KVCache((1, hq, hkv, d, 4), [wl.cfg(0)], [n0], codebooks=[float(x) for x in books.astype(np.float16)])
    k = (rng.standard_normal((n0, hkv, d)) * 2).astype(np.float16)
    v = np.full((n0, hkv, d), 65504.0, np.float16)
    v[:, :, ::3] = -65504.0
    c.append_prompt(dev(k), dev(v))
    q, kt, _ = drafts(wl, rng, n)
    vt = np.broadcast_to(v[0], (1, n, hkv, d)).copy()
    mask, _ = trees(rng, 1, n)
    got = attend(c, q, kt, vt, mask).astype(np.float64)
    want = np.broadcast_to(v[0, 0].astype(np.float64), got.shape)
    # the weights' roundings (u), the values' (3 u, uniform 4-bit), the result's (u)
    assert np.all(np.abs(got - want) <= 5 * U * 65504), np.abs(got).max()


def test_one_weight_rounded_up_takes_no_value_past_the_end():
    """A cached token whose weight is just over twice a node's, in steps of 2^-16 or so: where its fp16
    probability is rounded up by half a step, the quotient lies above what it is a mean of."""
    from paper_2609_07966_amd.cache import KVCache
    n, hq, hkv, d = 64, 8, 2, 64
    c = KVCache((1, hq, hkv, d, 4), [{"method": "fp16"}], [1])
    k, v = np.zeros((1, hkv, d), np.float16), np.full((1, hkv, d), 65504.0, np.float16)
    k[..., :2] = 1
    c.append_prompt(dev(k), dev(v))
    q, kt = np.zeros((1, n, hq, d), np.float16), np.zeros((1, n, hkv, d), np.float16)
    q[..., 0] = 8 * np.log(2)  # the logit of the cached token is about log 2, that of the nodes 0
    q[0, :, :, 1] = (np.arange(n * hq).reshape(n, hq) - 64) * 2.0 ** -14
    mask = (np.uint64(1) << np.arange(n, dtype=np.uint64))[None]
    got = attend(c, q, kt, np.full((1, n, hkv, d), 65504.0, np.float16), mask).astype(np.float64)
    assert np.all(np.abs(got - 65504) <= 2 * U * 65504), got.max()


def ratio_books(key, value):
    """Codebooks for 2, 3 and 4 bits whose largest entries are `key` and `value`: {bits: (keys, values)}, flat."""
    books = {b: tuple((np.linspace(-1, 1, 1 << b) * top).astype(np.float16).astype(np.float32) for top in (key, value))
             for b in (2, 3, 4)}
    return books, [float(x) for b in (2, 3, 4) for cb in books[b] for x in cb]


@pytest.mark.parametrize("key,value", [(1.0, 1.0), (1.0625, 1.1875), (3.0, 2.5), (0.5, 1.5), (700.0, 1.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_kvquant_thresholds_at_the_end_of_fp16(d, key, value):
    """Codebooks that go past their thresholds (an entry of 1.19 stands for 1.19 times it) and thresholds and
    scales up to the last finite fp16 value: what a code stands for may then lie past fp16's end."""
    from oracle.sequence import Sequence
    from paper_2609_07966_amd.cache import KVCache
    rng = np.random.default_rng(36)
    lens, hq, hkv, n = [90, 300, 1100], 4, 2, 6
    cfgs = [{"method": "kvq", "bits": b, "outlier_bp": bp} for b, bp in ((4, 100), (3, 400), (2, 0))]
    books, flat = ratio_books(key, value)
    t = sum(lens)
    k, v = (rng.standard_normal((t, hkv, d)).astype(np.float16) for _ in range(2))
    # tokens of all sizes, a third of them up to the last finite value; four channels of such keys
    size = np.where(rng.random((t, hkv, 1)) < 1 / 3, 65504.0, 10.0 ** rng.integers(-2, 4, (t, hkv, 1)))
    v = (rng.uniform(-1, 1, (t, hkv, d)) * size).astype(np.float16)
    v[0] = 65504
    k[..., :4] = (rng.uniform(-1, 1, (t, hkv, 4)) * 65504).astype(np.float16)
    c = KVCache((3, hq, hkv, d, 4), cfgs, lens, codebooks=flat)
    c.append_prompt(dev(k), dev(v))
    q, kt, vt = (rng.standard_normal((3, n, h, d)).astype(np.float16) for h in (hq, hkv, hkv))
    q = (q / max(1.0, key)).astype(np.float16)
    q[..., :4] = (rng.standard_normal((3, n, hq, 4)) * 2.0 ** -13 / max(1.0, key)).astype(np.float16)
    mask, _ = trees(rng, 3, n)
    mask[:, 0] = 0
    got = attend(c, q, kt, vt, mask).astype(np.float64)
    row = past = 0
    for s, n0 in enumerate(lens):
        seq = Sequence(cfgs[s], k[row:row + n0], v[row:row + n0], hq, codebooks=books)
        keys, vals = [x["eff"] for x in seq.kq], [x["eff"] for x in seq.vq]
        # a decoded value's own rounding; near 0 half a subnormal step, of values in units of the codebook's largest
        # entry (a power of two at most twice it)
        err = lambda x, top: U * np.abs(x) + 2.0 ** -25 * max(1.0, 2 * top)
        past += sum(float(np.abs(x).max()) > 65520 for x in vals)
        bounded(keys, vals, [err(x, key) for x in keys], [err(x, value) for x in vals], q[s], kt[s], vt[s], mask[s], got[s])
        row += n0
    assert value <= 1 or past > 0


# ---- acceptance ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("max_new", [1, 5, 6, 7, 8])
def test_accept_ends_at_max_new_under_every_method(d, max_new):
    """Equal paths leave equal numbers of tokens in a mixed batch, whatever their methods round their room
    up to, in one acceptance or over several; and every kv head holds them."""
    import torch
    names, n0 = CONFIGS + ["KVQ4"], 61
    wl = workload(names, [n0] * 6, 4, 2, d)
    cfg = wl.cfg
    wl.cfg = lambda s: dict(cfg(s), outlier_bp=5000) if s == 5 else cfg(s)
    rng = np.random.default_rng(37)
    _, kt, vt = drafts(wl, rng, 12)
    kt *= 50  # (nearly every key past its threshold: the outlier pools fill up)
    path = np.tile(np.arange(12, dtype=np.int32), (6, 1))
    counts = torch.zeros(6, dtype=torch.int32, device="cuda")
    state = []
    for rounds in ([12], [2, 3, 12, 12]):
        c, _ = admitted(wl, max_new)
        at = 0
        for m in rounds:
            c.tree_accept(dev(kt), dev(vt), dev(np.roll(path, -at, 1)), dev(np.full(6, m, np.int32)), counts)
            at = min(at + m, max_new)
            assert counts.tolist() == [n0 + at] * 6
        assert at == max_new
        assert all(c.counts(s, h)[0] == n0 + max_new for s in range(6) for h in range(2))
        state.append([exports(c, s, h, wl.cfg(s)["method"]) for s in range(6) for h in range(2)])
    assert all(same_state(a, b) for a, b in zip(*state))


def configured(names, extra, lens, hq, hkv, d):
    wl = workload(names, lens, hq, hkv, d)
    cfg = wl.cfg
    wl.cfg = lambda s: {"method": "kvq", "bits": extra[s][0], "outlier_bp": extra[s][1]} if s in extra else cfg(s)
    return wl


@pytest.mark.parametrize("d", [64, 128])
def test_decode_steps_after_an_acceptance(d):
    """The decode step reads what acceptance wrote through other words than the tree attention does (an
    outlier's difference from its code): steps after it are bit for bit those of a twin that appended the same
    tokens one decode step at a time, with several outliers a token, fewer than there are slots for, and none.
    The first beam of each pair accepts over slots that held other tokens before it took the second's state."""
    import torch
    each = CONFIGS + ["KVQ4"] * 4
    extra = {5: (4, 400), 6: (3, 250), 7: (2, 5000), 8: (4, 0)}
    lens = [70, 60, 50, 33, 126, 90, 65, 40, 64]
    wl = configured([x for x in each for _ in range(2)], {2 * i + w: x for i, x in extra.items() for w in range(2)},
                    [x for x in lens for _ in range(2)], 8, 2, d)
    s, n, m = wl.n_seqs, 10, 7
    rng = np.random.default_rng(38)
    q, kt, vt = drafts(wl, rng, n)
    vt[:, 4, :, : d // 2] = 0
    vt[:, 5] = 1  # ties: nothing over the scale
    kt[:, 6] *= 30
    path = np.tile(np.array([6, 4, 0, 5, 9, 4, 2], np.int32), (s, 1))
    a, _ = admitted(wl, 24, same=2)
    b, _ = admitted(wl, 24, same=2)
    a.tree_accept(dev((kt * -3).astype(np.float16)), dev((vt[:, ::-1] * 5).astype(np.float16)), dev(path),
                  dev(np.tile(np.array([m, 0], np.int32), s // 2)))
    a.reorder(dev(np.ones(s, np.int32)), 2)
    a.tree_accept(dev(kt), dev(vt), dev(path), dev(np.full(s, m, np.int32)))
    out_a, out_b = (torch.empty((s, 8, d), dtype=torch.float32, device="cuda") for _ in range(2))
    for node in path[0]:
        b.step(dev(kt[:, node]), dev(vt[:, node]), dev(q[:, 0]), out_b)
    for t in range(4):
        one = [dev(x) for x in step_inputs(wl, t)]
        a.step(*one, out_a)
        b.step(*one, out_b)
        assert bool(torch.isfinite(out_a).all())
        for i in range(s):
            assert torch.equal(out_a[i], out_b[i]), (t, i, wl.cfg(i))


# ---- streams ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("side", [True, False])
def test_cache_calls_follow_the_current_stream(side):
    """rope and beam_select run on the current stream and the cache's calls on the stream it was made with:
    with two different ones, inputs still on their way and outputs read at once, a round gives what it gives
    on one stream."""
    import torch
    from paper_2609_07966_amd import decoding
    wl = workload(["FP16", "FP16", "KVQ4", "KVQ4", "UQ4-g64", "UQ4-g64"], [200, 200, 90, 90, 150, 150], 8, 2, 128)
    s, n, m = 6, 8, 3
    rng = np.random.default_rng(39)
    inv_freq = dev((10000.0 ** (-np.arange(64) / 64)).astype(np.float32))
    rounds = []
    for _ in range(3):
        q, kt, vt = drafts(wl, rng, n)
        mask, _ = trees(rng, s, n)
        rounds.append([dev(x) for x in (q, kt, vt, mask.view(np.int64), np.tile(rng.integers(0, 1000, n), s)[None].astype(np.int32),
                                        rng.integers(0, n, (s, m)).astype(np.int32), rng.integers(0, m + 1, s).astype(np.int32),
                                        rng.standard_normal((s // 2, 2, 4001)).astype(np.float32))])
    scores = torch.zeros((s // 2, 2), device="cuda")
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()

    def go(c, slow):
        results = []
        for x in rounds:
            held = [torch.zeros_like(t) for t in x]
            if slow:
                torch.cuda._sleep(4000000)  # some ms, before the inputs are there
            for dst, src in zip(held, x):
                dst.copy_(src)
            q, kt, vt, mask, pos, path, n_path, logits = held
            qr, kr = decoding.rope([q.view(s * n, 8, 128), kt.view(s * n, 2, 128)], pos, inv_freq)
            qr, kr = qr.view(q.shape), kr.view(kt.shape)
            out = c.tree_attention(qr, kr, vt, mask)
            results.append(out * 1)  # (read at once, on the current stream)
            counts = torch.zeros(s, dtype=torch.int32, device="cuda")
            c.tree_accept(kr, vt, path, n_path, counts)
            results.append(counts * 1)
            _, parent, _ = decoding.beam_select(logits, scores, 2)
            c.reorder(parent.view(-1), 2)
            del held, q, kt, vt, mask, qr, kr, out, parent
        return results

    with torch.cuda.stream(a):
        one, _ = admitted(wl, 40, same=2, stream=a)
        want = go(one, False)
    torch.cuda.synchronize()
    two, _ = admitted(wl, 40, same=2, stream=a if side else torch.cuda.default_stream())
    torch.cuda.synchronize()
    with torch.cuda.stream(b):
        got = go(two, True)
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x, y)
    for i in range(s):
        for h in range(2):
            assert same_state(exports(one, i, h, wl.cfg(i)["method"]), exports(two, i, h, wl.cfg(i)["method"]))


def test_cache_calls_captured_on_another_stream():
    """Captured under a stream that is not the cache's: the cache's stream joins the capture and comes back."""
    import torch
    wl = workload(["FP16", "KVQ3", "UQ4-g64"], [300, 90, 150], 8, 2, 64)
    rng = np.random.default_rng(40)
    q, kt, vt = drafts(wl, rng, 6)
    mask, _ = trees(rng, 3, 6)
    inputs = [dev(x) for x in (q, kt, vt, mask.view(np.int64))]
    path, n_path = dev(np.tile(np.arange(6, dtype=np.int32), (3, 1))), dev(np.array([2, 0, 3], np.int32))
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        eager, _ = admitted(wl, 40, stream=own)
        twin, _ = admitted(wl, 40, stream=own)
    torch.cuda.synchronize()
    out = torch.zeros_like(inputs[0])
    ws = eager.tree_workspace(6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        twin.tree_attention(*inputs, out=out, workspace=ws)
        twin.tree_accept(inputs[1], inputs[2], path, n_path)
    for _ in range(4):
        want = eager.tree_attention(*inputs)
        eager.tree_accept(inputs[1], inputs[2], path, n_path)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    for i in range(3):
        assert same_state(exports(eager, i, 1, wl.cfg(i)["method"]), exports(twin, i, 1, wl.cfg(i)["method"]))


def test_a_refused_call_leaves_a_capture_whole():
    import torch
    from paper_2609_07966_amd import _lib
    wl = workload(["FP16"], [100], 4, 2, 64)
    rng = np.random.default_rng(41)
    q, kt, vt = drafts(wl, rng, 4)
    inputs = [dev(x) for x in (q, kt, vt, np.ones((1, 4), np.int64))]
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        c, _ = admitted(wl, 4, stream=own)
        want = c.tree_attention(*inputs)
    torch.cuda.synchronize()
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        with pytest.raises(_lib.MkvError):
            c.reorder(torch.zeros(1, dtype=torch.int32, device="cuda"), 33)
        c.tree_attention(*inputs, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
