"""Drafted trees over a mixed cache (mkv_tree_attention, mkv_tree_accept) against the float64 oracle's
cache contents, and the reordering of beams (mkv_cache_reorder) against the states before it.

Tolerance of the attention, per output value, from its roundings (u = 2^-11, half an fp16 step relative
to the value): the result itself (u |o|); probabilities, rounded to fp16 before they weigh values
(u A, A = sum p |v| over the row); quantized values, rounded when they are decoded (u A; uniform 4-bit
also rounds the step, u (|v| + |min|) <= 2 u (range) a value: 3 u A' with A' = sum p (|v| + |min|)); and quantized keys,
whose logit moves by at most dl = c u sum |q k| / sqrt(d) (c = 1, uniform 4-bit 3 on |k| + |min|), which moves
the result by at most (exp(2 dl) - 1) A.  Sums in float32 add some 1e-6 A, covered by 1e-5 A.  And in the
mean, rounding errors being independent, the relative 2-norm of the error stays below 4 u."""
import numpy as np
import pytest

from workloads import make_workload, prompt_kv, prompt_q, step_inputs

pytestmark = pytest.mark.gpu
U = 2.0 ** -11


@pytest.fixture(autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import os
    import sys
    sys.path.insert(0, os.path.dirname(__file__))
    from paper_2609_07966_amd import _lib
    _lib.lib()


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def workload(names, lens, hq=8, hkv=2, d=128, seed=3):
    return make_workload("custom", seed=seed, n_seqs=len(lens), n_q_heads=hq, n_kv_heads=hkv, head_dim=d,
                         prompt_lens=lens, steps=1, config_ids=names)


def admitted(wl, max_new, same=1, stream=None):
    """A cache after its prompts; same: groups of that many sequences share their first one's prompt."""
    from gpu_harness import _window_block, oracle_codebooks
    from paper_2609_07966_amd.cache import KVCache
    cfgs = [wl.cfg(s) for s in range(wl.n_seqs)]
    books, flat = oracle_codebooks(wl)
    c = KVCache((wl.n_seqs, wl.n_q_heads, wl.n_kv_heads, wl.head_dim, max_new), cfgs, wl.prompt_lens,
                codebooks=list(flat), stream=stream)
    kv = [prompt_kv(wl, s - s % same) for s in range(wl.n_seqs)]
    c.append_prompt(dev(np.concatenate([a for a, _ in kv])), dev(np.concatenate([b for _, b in kv])))
    hq = [prompt_q(wl, s - s % same) for s in range(wl.n_seqs) if cfgs[s]["method"] == "h2o"]
    if hq:
        c.h2o_prefill(dev(np.concatenate(hq)))
    rq = [_window_block(wl, s - s % same, 32) for s in range(wl.n_seqs) if cfgs[s]["method"] == "rocket"]
    if rq:
        c.snap_prefill(dev(np.concatenate(rq)))
    return c, books


def trees(rng, s, n):
    """Random ancestor masks [S][N] and parents."""
    mask, parent = np.zeros((s, n), np.uint64), np.full((s, n), -1)
    for i in range(s):
        for j in range(n):
            p = int(rng.integers(max(-1, j - 5), j)) if j else -1
            parent[i, j] = p
            mask[i, j] = (mask[i, p] if p >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(j))
    return mask, parent


def drafts(wl, rng, n):
    shape = lambda h: (wl.n_seqs, n, h, wl.head_dim)
    return [rng.standard_normal(shape(h)).astype(np.float16) for h in (wl.n_q_heads, wl.n_kv_heads, wl.n_kv_heads)]


class Held:
    """What a cache holds of one sequence, from the oracle, in float64: per kv head keys, values and the
    magnitudes that their roundings are relative to."""

    def __init__(self, wl, books, s, extra_k=None, extra_v=None):
        from oracle import uniform
        from oracle.sequence import Sequence
        kp, vp = prompt_kv(wl, s)
        seq = Sequence(wl.cfg(s), kp, vp, wl.n_q_heads, codebooks=books)
        self.keys, self.vals, self.kmag, self.vmag = [], [], [], []
        self.method = wl.cfg(s)["method"]
        for h in range(wl.n_kv_heads):
            k, v = kp[:, h], vp[:, h]
            if extra_k is not None:
                k, v = np.vstack([k, extra_k[:, h]]), np.vstack([v, extra_v[:, h]])
            if self.method == "kvq":
                ke, ve = seq.kq[h]["eff"], seq.vq[h]["eff"]
                if extra_k is not None and len(extra_k):
                    ke = np.vstack([ke, seq._kvq_k(extra_k[:, h], h)["eff"]])
                    ve = np.vstack([ve, seq._kvq_v(extra_v[:, h])["eff"]])
            elif self.method == "uq":
                ke, ve = uniform.effective_keys(k, 4, 64), uniform.effective_values(v, 4, 64)
            else:
                ke, ve = k.astype(np.float64), v.astype(np.float64)
            self.keys.append(ke)
            self.vals.append(ve)
            km, vm = np.abs(ke), np.abs(ve)
            if self.method == "uq":
                for a in range(0, len(k) // 64 * 64, 64):
                    km[a:a + 64] += np.abs(k[a:a + 64].astype(np.float64).min(0))
                vm = vm + np.abs(v.astype(np.float64).reshape(len(v), -1, 64).min(2)).repeat(64, 1)
            self.kmag.append(km)
            self.vmag.append(vm)


def check(wl, held, s, q, kt, vt, mask, out, valid):
    """out [N][Hq][d] of sequence s; rows at or past `valid` are not looked at."""
    g, d = wl.group, wl.head_dim
    c = {"fp16": 0.0, "kvq": 1.0, "uq": 3.0}[held.method]
    num = den = 0.0
    for h in range(wl.n_kv_heads):
        for i in range(valid):
            seen = [j for j in range(valid) if int(mask[i]) >> j & 1]
            k = np.vstack([held.keys[h], kt[seen, h].astype(np.float64)])
            v = np.vstack([held.vals[h], vt[seen, h].astype(np.float64)])
            vm = np.vstack([held.vmag[h], np.abs(vt[seen, h].astype(np.float64))])
            qq = q[i, h * g:(h + 1) * g].astype(np.float64)
            z = qq @ k.T / np.sqrt(d)
            p = np.exp(z - z.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            ref, mag = p @ v, p @ vm
            dl = (np.abs(qq) @ held.kmag[h].T).max(1, keepdims=True) * c * U / np.sqrt(d)
            tol = U * np.abs(ref) + ((1 + c) * U + np.expm1(2 * dl) + 1e-5) * mag
            err = np.abs(out[i, h * g:(h + 1) * g].astype(np.float64) - ref)
            assert np.all(err <= tol), (s, h, i, float((err / tol).max()))
            num += float((err ** 2).sum())
            den += float((ref ** 2).sum())
    if den > 0:
        assert np.sqrt(num / den) <= 4 * U, (s, np.sqrt(num / den))


def run_and_check(wl, n, rng, valid=None, mask=None, edit=None, max_new=4):
    import torch
    c, books = admitted(wl, max_new)
    q, kt, vt = drafts(wl, rng, n)
    if mask is None:
        mask, _ = trees(rng, wl.n_seqs, n)
    if edit is not None:
        edit(q, kt, vt)
    nv = None if valid is None else torch.tensor(valid, dtype=torch.int32, device="cuda")
    out = torch.full((wl.n_seqs, n, wl.n_q_heads, wl.head_dim), 7.0, dtype=torch.float16, device="cuda")
    c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64)), out=out, n_valid=nv)
    got = out.cpu().numpy()
    for s in range(wl.n_seqs):
        v = n if valid is None else min(max(valid[s], 0), n)
        check(wl, Held(wl, books, s), s, q[s], kt[s], vt[s], mask[s], got[s], v)
        assert np.all(got[s, v:] == 7.0)
    return c, got


CONFIGS = ["FP16", "UQ4-g64", "KVQ4", "KVQ3", "KVQ2"]


@pytest.mark.parametrize("name", CONFIGS)
@pytest.mark.parametrize("hq,hkv,d,n", [(8, 2, 128, 4), (8, 2, 128, 8), (4, 4, 64, 16), (8, 4, 64, 33), (16, 2, 128, 9),
                                        (8, 1, 64, 64)])
def test_tree_attention(name, hq, hkv, d, n):
    # every number of rows a workgroup takes (16 to 128, and several workgroups), and odd ends of prompts
    wl = workload([name] * 3, [65, 300, 700], hq, hkv, d)
    run_and_check(wl, n, np.random.default_rng(5))


@pytest.mark.parametrize("name", CONFIGS)
def test_short_and_ragged(name):
    wl = workload([name] * 8, [1, 2, 31, 63, 64, 66, 127, 129], 4, 2, 128)
    rng = np.random.default_rng(6)
    run_and_check(wl, 1, rng)
    run_and_check(wl, 7, rng, valid=[7, 1, 0, 3, 7, -4, 9, 5])


@pytest.mark.parametrize("bits,bp", [(4, 400), (3, 250), (2, 5000), (4, 0)])
def test_outlier_budgets(bits, bp):
    """Several value outliers a token, half of all values, and none: attention, acceptance, reordering."""
    wl = workload(["KVQ4"] * 2, [130, 130], 4, 2, 128)
    wl.cfg = lambda s: {"method": "kvq", "bits": bits, "outlier_bp": bp}
    rng = np.random.default_rng(17)
    run_and_check(wl, 6, rng)
    a, _ = admitted(wl, 12, same=2)
    b, _ = admitted(wl, 12, same=2)
    _, kt, vt = drafts(wl, rng, 6)
    path = np.tile(np.array([5, 0, 3, 1, 2], np.int32), (2, 1))
    a.tree_accept(dev(kt), dev(vt), dev(path), dev(np.array([5, 0], np.int32)))
    import torch
    out = torch.empty((2, 4, 128), dtype=torch.float32, device="cuda")
    for node in path[0]:
        b.step(dev(kt[:, node]), dev(vt[:, node]), dev(drafts(wl, rng, 1)[0][:, 0]), out)
    for h in range(2):
        assert same_state(exports(a, 0, h, "kvq"), exports(b, 0, h, "kvq"))
    a.reorder(dev(np.array([0, 0], np.int32)), 2)
    for h in range(2):
        assert same_state(exports(a, 1, h, "kvq"), exports(b, 0, h, "kvq"))


def test_mixed_batch_and_splits():
    wl = workload(CONFIGS + ["FP16"], [3000, 1500, 900, 2047, 4100, 40], 8, 2, 128)
    run_and_check(wl, 12, np.random.default_rng(7))


def test_many_ragged_sequences():
    # more sequences than a wave has lanes, of which only some are split
    lens = [40 + 3 * (s % 9) for s in range(70)]
    for s, n in ((0, 900), (13, 2100), (63, 700), (64, 1500), (69, 1100)):
        lens[s] = n
    wl = workload([CONFIGS[s % 5] for s in range(70)], lens, 4, 2, 64)
    run_and_check(wl, 3, np.random.default_rng(20))


def test_masks():
    # empty words, words that name later nodes, nodes past the tree, and every node
    wl = workload(["FP16", "KVQ4", "UQ4-g64"], [100, 200, 300], 4, 2, 64)
    rng = np.random.default_rng(8)
    mask = rng.integers(0, 2 ** 63, size=(3, 10), dtype=np.uint64)
    mask[:, 0] = 0
    mask[:, 1] = np.uint64(0xFFFFFFFFFFFFFFFF)
    mask[:, 2] = np.uint64(0xFFFFFFFFFFFFFC00)
    run_and_check(wl, 10, rng, mask=mask)


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_unseen_nodes_reach_no_row(bad):
    # node 3's key and value are not finite; only the rows that attend to it may notice
    wl = workload(["FP16", "KVQ3"], [90, 200], 4, 2, 128)
    rng = np.random.default_rng(9)
    mask, _ = trees(rng, 2, 6)
    mask[:, 4:] &= ~np.uint64(8)
    mask[:, 3] |= np.uint64(8)
    import torch
    c, books = admitted(wl, 2)
    q, kt, vt = drafts(wl, rng, 6)
    vt[:, 3] = bad
    kt[:, 5] = np.float16(bad)
    mask[:, 5] = 0
    mask &= ~np.uint64(32)
    out = c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64))).cpu().numpy()
    for s in range(2):
        rows = [i for i in range(6) if not int(mask[s, i]) & 8]
        assert np.all(np.isfinite(out[s, rows])) and 3 not in rows
        assert not np.any(np.isfinite(out[s, 3]))
        clean = np.where(np.isfinite(vt), vt, 0).astype(np.float16)
        held = Held(wl, books, s)
        for i in rows:
            one = np.zeros(6, np.uint64)
            one[0] = mask[s, i]
            check(wl, held, s, q[s, i:i + 1], kt[s], clean[s], one, out[s, i:i + 1], 1) if not int(mask[s, i]) >> 1 else None
    # beyond n_valid nothing is read
    nv = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    again = c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64)), n_valid=nv).cpu().numpy()
    assert np.all(np.isfinite(again[:, :3]))


def test_unaligned_tensors_and_large_logits():
    import torch
    wl = workload(["FP16", "KVQ4", "UQ4-g64"], [257, 150, 130], 8, 2, 128)
    rng = np.random.default_rng(10)
    c, books = admitted(wl, 2)
    q, kt, vt = drafts(wl, rng, 5)
    q *= 20  # one or two keys carry a row's weight
    mask, _ = trees(rng, 3, 5)

    def odd(x):
        buf = torch.zeros(x.size + 1, dtype=torch.float16, device="cuda")
        view = buf[1:].view(x.shape)
        view.copy_(dev(x))
        return view
    aligned = c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64)))
    out = odd(np.zeros(q.shape, np.float16))
    c.tree_attention(odd(q), odd(kt), odd(vt), dev(mask.view(np.int64)), out=out)
    assert torch.equal(aligned, out)
    got = out.cpu().numpy()
    held = Held(wl, books, 0)  # fp16 rows: no rounding of keys, so the bound holds for any logits
    check(wl, held, 0, q[0], kt[0], vt[0], mask[0], got[0], 5)


@pytest.mark.parametrize("n", [1, 16, 64])
def test_many_small_weights(n):
    """One token has nearly all the weight and a value of 0; the output is the tail's, 2^-25.5 each, which
    the roundings above keep to u a value like any other."""
    from types import SimpleNamespace

    from paper_2609_07966_amd.cache import KVCache
    t, hq, hkv, d = 8192, 8, 2, 128
    c = KVCache((1, hq, hkv, d, 4), [{"method": "fp16"}], [t])
    k, v = np.zeros((t, hkv, d), np.float16), np.ones((t, hkv, d), np.float16)
    k[:, :, 0] = -25  # logits of 8 * -25 / sqrt(128)
    k[5], v[5] = 0, 0
    c.append_prompt(dev(k), dev(v))
    q = np.zeros((1, n, hq, d), np.float16)
    q[..., 0] = 8
    kt, vt = np.zeros((2, 1, n, hkv, d), np.float16)
    mask = np.zeros((1, n), np.uint64)
    got = c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64))).cpu().numpy()
    kk, vv = [k[:, h].astype(np.float64) for h in range(hkv)], [v[:, h].astype(np.float64) for h in range(hkv)]
    held = SimpleNamespace(method="fp16", keys=kk, vals=vv, kmag=kk, vmag=vv)
    check(SimpleNamespace(group=hq // hkv, head_dim=d, n_kv_heads=hkv), held, 0, q[0], kt[0], vt[0], mask[0], got[0], n)


def test_kvquant_thresholds_and_queries_of_all_sizes():
    """Channels whose prompt was 0 or tiny and whose accepted tokens are not (every value an outlier far past
    its threshold), a channel at the end of fp16, and rows of queries that are far apart in size.  Queries are
    small where keys are large, so that logits stay within some units."""
    from gpu_harness import oracle_codebooks
    wl = workload(["KVQ4", "KVQ3", "KVQ2"], [100, 100, 100], 4, 2, 64)
    from paper_2609_07966_amd.cache import KVCache
    cfgs = [wl.cfg(s) for s in range(3)]
    books, flat = oracle_codebooks(wl)
    from oracle.sequence import Sequence
    rng = np.random.default_rng(19)
    size = np.zeros(64)
    size[8:16], size[16:24], size[24:40], size[40:48] = 2.0 ** -22, 2.0 ** -9, 1.0, 300.0
    k = (rng.standard_normal((3, 100, 2, 64)) * size).astype(np.float16)
    v = rng.standard_normal((3, 100, 2, 64)).astype(np.float16)
    c = KVCache((3, 4, 2, 64, 8), cfgs, [100] * 3, codebooks=list(flat))
    c.append_prompt(dev(k.reshape(300, 2, 64)), dev(v.reshape(300, 2, 64)))
    n = 4
    kt, vt = (rng.standard_normal((2, 3, n, 2, 64))).astype(np.float16)
    kt[..., :4] *= 1000
    kt[:, 0, :, 60] = 65504
    path = np.tile(np.arange(n, dtype=np.int32), (3, 1))
    c.tree_accept(dev(kt), dev(vt), dev(path), dev(np.full(3, n, np.int32)))
    q = rng.standard_normal((3, n, 4, 64))
    q[..., :4] *= 2.0 ** -9
    q[..., 40:48] *= 2.0 ** -8
    q[..., 60] = 2.0 ** -16
    q[:, 0] *= 2.0 ** -6
    q[:, 2] *= 2
    q = q.astype(np.float16)
    mask = np.zeros((3, n), np.uint64)
    got = c.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64))).cpu().numpy()
    from types import SimpleNamespace
    for s in range(3):
        seq = Sequence(cfgs[s], k[s], v[s], 4, codebooks=books)
        keys, vals = [], []
        for h in range(2):
            keys.append(np.vstack([seq.kq[h]["eff"], seq._kvq_k(kt[s, :, h], h)["eff"]]))
            vals.append(np.vstack([seq.vq[h]["eff"], seq._kvq_v(vt[s, :, h])["eff"]]))
        held = SimpleNamespace(method="kvq", keys=keys, vals=vals, kmag=[np.abs(x) for x in keys], vmag=[np.abs(x) for x in vals])
        for i in (0, 1, 2, 3):
            one = np.zeros(1, np.uint64)
            check(wl, held, s, q[s, i:i + 1], kt[s, :1], vt[s, :1], one, got[s, i:i + 1], 1)


def exports(c, s, h, method):
    from paper_2609_07966_amd import _lib
    kinds = {"fp16": ["counts", "positions"], "uq": ["counts", "codes_k", "codes_v", "scales_k", "scales_v"],
             "kvq": ["counts", "codes_k", "codes_v", "outliers_k", "outliers_v", "scales_k", "scales_v"],
             "h2o": ["counts", "positions", "scores"], "rocket": ["counts", "positions", "topk", "channels"]}
    # (a small buffer: the wrapper's own default is cleared on every call)
    return {k: np.frombuffer(_lib.mkv_export(c.h, s, h, k, cap=1 << 19), np.uint8) for k in kinds[method]}


def same_state(a, b):
    return a.keys() == b.keys() and all(np.array_equal(a[k], b[k]) for k in a)


@pytest.mark.parametrize("d", [64, 128])
def test_accept_is_the_decode_append(d):
    """Accepted paths against the same tokens appended one decode step at a time, bit for bit."""
    import torch
    names, lens = CONFIGS, [70, 60, 50, 33, 126]
    wl = workload(names, lens, 4, 2, d)
    rng = np.random.default_rng(11)
    a, _ = admitted(wl, 24)
    b, _ = admitted(wl, 24)
    n, m = 12, 9
    took = [9, 7, 9, 0, 5]
    q, kt, vt = drafts(wl, rng, n)
    kt *= 3
    path = np.stack([rng.permutation(n)[:m] for _ in names]).astype(np.int32)
    path[2, 6] = 12  # ends this path at six tokens
    path[1, 3] = path[1, 2]  # a node twice
    counts = torch.zeros(len(names), dtype=torch.int32, device="cuda")
    a.tree_accept(dev(kt), dev(vt), dev(path), dev(np.array(took, np.int32)), counts)
    real = [9, 7, 6, 0, 5]
    assert counts.tolist() == [x + y for x, y in zip(lens, real)]
    out = torch.empty((len(names), 4, d), dtype=torch.float32, device="cuda")
    for s in range(len(names)):
        # the twin appends sequence s's path to all of its sequences; only sequence s is compared
        twin, _ = admitted(wl, 24)
        for t in range(real[s]):
            node = path[s, t]
            twin.step(dev(kt[:, node]), dev(vt[:, node]), dev(q[:, 0]), out)
        for h in range(2):
            assert same_state(exports(a, s, h, wl.cfg(s)["method"]), exports(twin, s, h, wl.cfg(s)["method"])), (s, h)
    # the cache goes on: another round, and a decode step, as the oracle's cache would
    mask, _ = trees(rng, len(names), n)
    got = a.tree_attention(dev(q), dev(kt), dev(vt), dev(mask.view(np.int64))).cpu().numpy()
    from gpu_harness import oracle_codebooks
    books, _ = oracle_codebooks(wl)
    for s in range(len(names)):
        p = path[s, :real[s]]
        check(wl, Held(wl, books, s, kt[s, p], vt[s, p]), s, q[s], kt[s], vt[s], mask[s], got[s], n)
    kn, vn, qn = step_inputs(wl, 0)
    a.step(dev(kn), dev(vn), dev(qn), out)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out).all())
    del b


def test_accept_drops_what_has_no_room():
    import torch
    wl = workload(["FP16", "KVQ4", "UQ4-g64"], [61, 61, 61], 4, 2, 64)
    rng = np.random.default_rng(12)
    c, _ = admitted(wl, 3)  # capacities: 64 slots each
    _, kt, vt = drafts(wl, rng, 8)
    path = np.tile(np.arange(8, dtype=np.int32), (3, 1))
    counts = torch.zeros(3, dtype=torch.int32, device="cuda")
    c.tree_accept(dev(kt), dev(vt), dev(path), dev(np.full(3, 8, np.int32)), counts)
    assert counts.tolist() == [64, 64, 64]
    before = [exports(c, s, 1, wl.cfg(s)["method"]) for s in range(3)]
    c.tree_accept(dev(kt), dev(vt), dev(path), dev(np.full(3, 8, np.int32)), counts)
    assert counts.tolist() == [64, 64, 64]
    assert all(same_state(before[s], exports(c, s, 1, wl.cfg(s)["method"])) for s in range(3))


@pytest.mark.parametrize("name", CONFIGS + ["H2O-20", "H2O-50", "Rocket-1024", "Rocket-8x"])
@pytest.mark.parametrize("max_new,steps,width", [(8, 6, 4), (700, 40, 3), (90, 70, 8)])
def test_reorder(name, max_new, steps, width):
    """Beams with tails of their own take their parents' states in place: exports equal, and a step of
    equal inputs equals, bit for bit, what the parents' states gave in a twin that stayed in order."""
    import torch
    if max_new == 700 and name not in ("FP16", "KVQ3", "H2O-50", "Rocket-8x", "UQ4-g64"):
        pytest.skip("one of a method's configurations is enough at this size")
    wl = workload([name] * (2 * width), [150] * width + [201] * width, 4, 2, 64 if width == 4 else 128)
    method = wl.cfg(0)["method"]
    rng = np.random.default_rng(13)
    a, _ = admitted(wl, max_new, same=width)
    b, _ = admitted(wl, max_new, same=width)
    out_a = torch.empty((2 * width, 4, wl.head_dim), dtype=torch.float32, device="cuda")
    out_b = torch.empty_like(out_a)
    for t in range(steps):
        kn, vn, qn = (dev(x) for x in step_inputs(wl, t))
        a.step(kn, vn, qn, out_a)
        b.step(kn, vn, qn, out_b)
    for parent in ([(w + 1) % width for w in range(width)], [int(x) for x in rng.integers(0, width, width)]):
        full = np.array(parent + [width - 1] + [0] * (width - 2) + [77], np.int32)  # 77: stays
        eff = list(parent) + [width - 1] + [0] * (width - 2) + [width - 1]
        before = {(s, h): exports(a, s, h, method) for s in range(2 * width) for h in range(2)}
        a.reorder(dev(full), width)
        for s in range(2 * width):
            src = s // width * width + eff[s]
            for h in range(2):
                assert same_state(exports(a, s, h, method), before[src, h]), (s, src, h)
        if parent[0] == 1:  # the twin still has the parents' states
            one = [dev(np.broadcast_to(x[:1], x.shape)) for x in step_inputs(wl, 777)]
            a.step(*one, out_a)
            b.step(*one, out_b)
            ga, gb = out_a.cpu().numpy(), out_b.cpu().numpy()
            for s in range(2 * width):
                assert np.array_equal(ga[s], gb[s // width * width + eff[s]]), s


def test_reorder_after_paths_of_different_lengths():
    import torch
    wl = workload(["KVQ2"] * 3 + ["UQ4-g64"] * 3 + ["FP16"] * 3, [100] * 9, 4, 2, 64)
    rng = np.random.default_rng(14)
    c, _ = admitted(wl, 80, same=3)
    _, kt, vt = drafts(wl, rng, 64)
    path = np.tile(np.arange(64, dtype=np.int32), (9, 1))
    c.tree_accept(dev(kt), dev(vt), dev(path), dev(np.array([0, 64, 5, 40, 3, 0, 1, 2, 61], np.int32)))
    before = {(s, h): exports(c, s, h, wl.cfg(s)["method"]) for s in range(9) for h in range(2)}
    parent = [1, 2, 0, 2, 0, 0, 2, 2, 1]
    c.reorder(dev(np.array(parent, np.int32)), 3)
    for s in range(9):
        for h in range(2):
            assert same_state(exports(c, s, h, wl.cfg(s)["method"]), before[s // 3 * 3 + parent[s], h]), (s, h)
    # and tokens go on behind the new counts
    c.tree_accept(dev(kt), dev(vt), dev(path), dev(np.full(9, 7, np.int32)))
    for s in range(9):
        assert c.counts(s, 0)[0] == before[s // 3 * 3 + parent[s], 0]["counts"].view(np.int32)[0] + 7
    torch.cuda.synchronize()


def test_rounds_together_and_replayed():
    """A verification round as it is used (rotate, attend, accept, fork the best), eager and as a captured
    graph replayed several times with eager work between: bit for bit the same."""
    import torch
    from paper_2609_07966_amd import decoding
    wl = workload(["FP16", "FP16", "KVQ4", "KVQ4", "UQ4-g64", "UQ4-g64"], [200, 200, 90, 90, 150, 150], 8, 2, 128)
    s, n, m = 6, 8, 3
    rng = np.random.default_rng(15)
    stream = torch.cuda.Stream()
    inv_freq = dev((10000.0 ** (-np.arange(64) / 64)).astype(np.float32))
    rounds = []
    for _ in range(4):
        q, kt, vt = drafts(wl, rng, n)
        mask, _ = trees(rng, s, n)
        rounds.append([dev(x) for x in (q, kt, vt, mask.view(np.int64), np.tile(rng.integers(0, 1000, n), s)[None].astype(np.int32),
                                        rng.integers(0, n, (s, m)).astype(np.int32), rng.integers(0, m + 1, s).astype(np.int32),
                                        rng.integers(0, 2, s).astype(np.int32))])
    torch.cuda.synchronize()

    def go(c, x, out, ws, rot):
        q, kt, vt, mask, pos, path, n_path, parent = x
        decoding.rope([q.view(s * n, 8, 128), kt.view(s * n, 2, 128)], pos, inv_freq,
                      out=[rot[0].view(s * n, 8, 128), rot[1].view(s * n, 2, 128)])
        c.tree_attention(rot[0], rot[1], vt, mask, out=out, workspace=ws)
        c.tree_accept(rot[1], vt, path, n_path)
        c.reorder(parent, 2)

    def buffers(c):
        return (torch.zeros((s, n, 8, 128), dtype=torch.float16, device="cuda"), c.tree_workspace(n),
                [torch.empty((s, n, h, 128), dtype=torch.float16, device="cuda") for h in (8, 2)])

    with torch.cuda.stream(stream):
        eager, _ = admitted(wl, 40, same=2, stream=stream)
        out, ws, rot = buffers(eager)
        want = []
        for x in rounds:
            go(eager, x, out, ws, rot)
            want.append(out.clone())
        captured, _ = admitted(wl, 40, same=2, stream=stream)
        out2, ws2, rot2 = buffers(captured)
        held = [x.clone() for x in rounds[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        go(captured, held, out2, ws2, rot2)
    for x, w in zip(rounds, want):
        for dst, src in zip(held, x):
            dst.copy_(src)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out2, w)
    for i in range(s):
        for h in range(2):
            assert same_state(exports(eager, i, h, wl.cfg(i)["method"]), exports(captured, i, h, wl.cfg(i)["method"]))


def test_refusals():
    import torch
    from paper_2609_07966_amd import _lib as L
    wl = workload(["FP16", "H2O-20", "Rocket-1024"], [100, 100, 100], 4, 2, 64)
    c, _ = admitted(wl, 4)
    rng = np.random.default_rng(16)
    q, kt, vt = (dev(x) for x in drafts(wl, rng, 4))
    mask = torch.ones((3, 4), dtype=torch.int64, device="cuda")

    def status(fn, *a, **k):
        try:
            fn(*a, **k)
        except L.MkvError as e:
            return e.status
        return 0
    assert status(c.tree_attention, q, kt, vt, mask) == 5
    path = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    assert status(c.tree_accept, kt, vt, path, path[:, 0].contiguous()) == 5
    assert status(c.reorder, torch.zeros(3, dtype=torch.int32, device="cuda"), 3) == 1  # three methods
    wl = workload(["FP16", "FP16"], [4000, 4000], 4, 2, 64)
    c, _ = admitted(wl, 4)
    q, kt, vt = (dev(x) for x in drafts(wl, rng, 4))
    mask = torch.ones((2, 4), dtype=torch.int64, device="cuda")
    for bad in (dict(q=q[:, :3]), dict(k=kt.float()), dict(mask=mask.int()), dict(v=vt.transpose(0, 1)),
                dict(n_valid=torch.ones(3, dtype=torch.int32, device="cuda")), dict(out=q.float()), dict(q=q.cpu())):
        with pytest.raises(ValueError):
            c.tree_attention(**{**dict(q=q, k=kt, v=vt, mask=mask), **bad})
    need = L.mkv_tree_workspace(c.h, 4)
    assert need > 0
    assert status(c.tree_attention, q, kt, vt, mask, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")) == 2
    assert status(c.tree_attention, q, kt, vt, mask, workspace=torch.empty(need + 1, dtype=torch.uint8, device="cuda")[1:]) == 1
    assert status(L.mkv_tree_workspace, c.h, 65) == 1 and status(L.mkv_tree_workspace, c.h, 0) == 1
    par = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert status(c.reorder, par, 0) == 1 and status(c.reorder, par, 33) == 1
    with pytest.raises(ValueError):
        c.reorder(par.long(), 2)
    # between the calls of a step none of them may come
    out = torch.empty((2, 4, 64), dtype=torch.float32, device="cuda")
    c.append(kt[:, 0].contiguous(), vt[:, 0].contiguous())
    assert status(c.tree_attention, q, kt, vt, mask) == 4
    assert status(c.tree_accept, kt, vt, torch.zeros((2, 1), dtype=torch.int32, device="cuda"), par) == 4
    assert status(c.reorder, par, 2) == 4
    c.attention(q[:, 0].contiguous(), out)
    assert status(c.tree_attention, q, kt, vt, mask) == 0
    torch.cuda.synchronize()
