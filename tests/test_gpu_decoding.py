"""Rotary positions (mkv_rope) and beam selection (mkv_beam_select) against float64, on the GPU."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_07966_amd import _lib
    _lib.lib()


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


# ---- rotary positions --------------------------------------------------------------------------------

def turned(x, pos, inv_freq, sections, layout, inverse):
    """x [rows][heads][d] -> float64."""
    y = x.astype(np.float64)
    rot, h = 2 * len(inv_freq), len(inv_freq)
    axis = np.repeat(np.arange(len(sections)), sections)
    t = pos[axis].T.astype(np.float64) * inv_freq.astype(np.float64) * (-1 if inverse else 1)
    c, s = np.cos(t)[:, None], np.sin(t)[:, None]
    a, b = (y[..., :h], y[..., h:rot]) if layout == "halves" else (y[..., 0:rot:2], y[..., 1:rot:2])
    a, b = a * c - b * s, b * c + a * s
    if layout == "halves":
        y[..., :h], y[..., h:rot] = a, b
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = a, b
    return y


def close(got, ref, x):
    """Half an fp16 step of the result (an fp16 subnormal's half step near 0), and sines and cosines off by
    at most 2^-18 (the hardware's 2^-20 and the angle's own rounding in turns, 2 pi 2^-25) times the
    pair's two values."""
    big = np.abs(x.astype(np.float64)).max(-1, keepdims=True)
    tol = 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2 * 2.0 ** -18 * big
    err = np.abs(got.astype(np.float64) - ref)
    assert np.all(err <= tol), float((err / tol).max())


def freqs(n):
    return (10000.0 ** (-np.arange(n) / n)).astype(np.float32)


def test_rope_many_rows_and_many_heads():
    """More rows than one launch has workgroups for (one a row here), in place; more heads than one grid
    row, with values behind rotary_dim."""
    import torch
    from paper_2609_07966_amd import decoding
    n, d = (1 << 24) + 3, 1022
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 36 GB of device memory")
    freq = torch.rand(d // 2, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda").view(1, n)
    x = torch.empty((n, 1, d), dtype=torch.float16, device="cuda")
    rows = torch.tensor([0, 1, (1 << 23) - 1, 1 << 23, (1 << 24) - 1, 1 << 24, n - 1], device="cuda")
    x[rows] = torch.randn((len(rows), 1, d), device="cuda").half()
    few = decoding.rope([x[rows]], pos[:, rows].contiguous(), freq)[0]
    decoding.rope([x], pos, freq, out=[x])
    assert torch.equal(x[rows], few)
    del x
    heads, d, half = 8192, 1024, 511
    xs = [torch.randn((1, heads, d), device="cuda").half() for _ in range(4)]
    p = torch.tensor([[12345]], dtype=torch.int32, device="cuda")
    ys = decoding.rope(xs, p, freq)
    t = (freq.double() * 12345).view(1, 1, half)
    for x, y in zip(xs, ys):
        a, b = x[..., :half].double(), x[..., half:2 * half].double()
        ref = torch.cat([a * t.cos() - b * t.sin(), b * t.cos() + a * t.sin()], -1)
        mag = (a ** 2 + b ** 2).sqrt().repeat(1, 1, 2)
        # the result's rounding (2^-11), and sine and cosine to 2^-19
        assert bool(((y[..., :2 * half].double() - ref).abs() <= 2.0 ** -11 * ref.abs() + 2.0 ** -18 * mag + 2.0 ** -25).all())
        assert torch.equal(y[..., 2 * half:], x[..., 2 * half:])


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("rows,heads,d,sections", [
    (1, (1,), 2, [1]), (5, (4, 4), 64, [32]), (33, (32, 8), 128, [16, 24, 24]), (700, (16, 2), 128, [32]),
    (3, (3, 1), 96, [7, 0, 9, 4]), (129, (2,), 64, [3, 6]), (17, (5, 2, 1, 7), 80, [40]), (2, (1,), 1024, [500, 12]),
    (300, (40,), 128, [0, 64])])
def test_rope(rows, heads, d, sections, layout):
    from paper_2609_07966_amd import decoding
    rng = np.random.default_rng(rows + d)
    xs = [rng.standard_normal((rows, h, d)).astype(np.float16) for h in heads]
    pos = rng.integers(-5, 100000, (len(sections), rows)).astype(np.int32)
    f = freqs(sum(sections))
    for inverse in (False, True):
        ys = decoding.rope([dev(x) for x in xs], dev(pos), dev(f), sections=sections, layout=layout, inverse=inverse)
        for x, y in zip(xs, ys):
            close(y.cpu().numpy(), turned(x, pos, f, sections, layout, inverse), x)


def test_rope_far_positions():
    from paper_2609_07966_amd import decoding
    rng = np.random.default_rng(1)
    pos = np.array([[0, 1, 2 ** 20 + 1, 2 ** 30 + 7, 2 ** 31 - 1, -2 ** 31]], np.int32)
    x = rng.standard_normal((6, 8, 128)).astype(np.float16)
    y = decoding.rope([dev(x)], dev(pos), dev(freqs(64)))[0].cpu().numpy()
    close(y, turned(x, pos, freqs(64), [64], "halves", False), x)
    assert np.array_equal(y[0], x[0])  # position 0 turns nothing


@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (72, 20)])
def test_rope_strides_and_in_place(d, rot):
    """q and k as slices of one projection, unaligned, in place; values between and behind them stay."""
    import torch
    from paper_2609_07966_amd import decoding
    rng = np.random.default_rng(2)
    rows, hq, hkv = 37, 6, 2
    base = rng.standard_normal((rows, (hq + 2 * hkv) * d + 5)).astype(np.float16)
    pos = rng.integers(0, 9000, (1, rows)).astype(np.int32)
    f = freqs(rot // 2)
    buf = torch.zeros(base.size + 1, dtype=torch.float16, device="cuda")
    qkv = buf[1:].view(base.shape)
    qkv.copy_(dev(base))
    q, k = qkv[:, :hq * d].view(rows, hq, d), qkv[:, hq * d:(hq + hkv) * d].view(rows, hkv, d)
    new = decoding.rope([q, k], dev(pos), dev(f))
    decoding.rope([q, k], dev(pos), dev(f), out=[q, k])
    got = qkv.cpu().numpy()
    cut = (hq + hkv) * d
    x = base[:, :cut].reshape(rows, hq + hkv, d)
    close(got[:, :cut].reshape(x.shape), turned(x, pos, f, [rot // 2], "halves", False), x)
    assert np.array_equal(got[:, cut:], base[:, cut:])
    assert torch.equal(new[0], q) and torch.equal(new[1], k)
    assert np.array_equal(got[:, :cut].reshape(x.shape)[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_rope_gradient(layout):
    """sum(w y) has the gradient that turns w back: against the formula and against differences."""
    from paper_2609_07966_amd import decoding
    rng = np.random.default_rng(3)
    rows, heads, d, sections = 4, 3, 32, [6, 6]
    x, w = (rng.standard_normal((rows, heads, d)).astype(np.float16) for _ in range(2))
    pos = rng.integers(0, 500, (2, rows)).astype(np.int32)
    f = freqs(12)
    g = decoding.rope([dev(w)], dev(pos), dev(f), sections=sections, layout=layout, inverse=True)[0].cpu().numpy()
    close(g, turned(w, pos, f, sections, layout, True), w)
    loss = lambda z: float((turned(z, pos, f, sections, layout, False) * w.astype(np.float64)).sum())
    for _ in range(20):
        at = tuple(int(rng.integers(n)) for n in x.shape)
        lo, hi = x.astype(np.float64), x.astype(np.float64)
        lo[at] -= 1.0
        hi[at] += 1.0
        # (the loss is linear: the difference is its slope); g is off by at most close()'s tolerance
        assert abs((loss(hi) - loss(lo)) / 2 - float(g[at])) <= 2.0 ** -11 * abs(float(g[at])) + 2.0 ** -17 * np.abs(w).max() + 1e-9


def test_rope_refusals_and_empty():
    import torch
    from paper_2609_07966_amd import decoding
    x = torch.zeros((3, 2, 64), dtype=torch.float16, device="cuda")
    pos = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    f = dev(freqs(32))
    for bad in (dict(xs=[x.float()]), dict(xs=[x, x[:2]]), dict(pos=pos.long()), dict(pos=pos[:, :2]), dict(inv_freq=f.double()),
                dict(sections=[31]), dict(layout="other"), dict(out=[x, x]), dict(xs=[x.transpose(0, 1)]),
                dict(out=[x[:, :1]]), dict(pos=pos.cpu()), dict(xs=[x[..., ::2]])):
        with pytest.raises(ValueError):
            decoding.rope(**{**dict(xs=[x], pos=pos, inv_freq=f), **bad})
    empty = decoding.rope([x[:0]], pos[:, :0], f)
    assert empty[0].shape == (0, 2, 64)


# ---- beam selection ------------------------------------------------------------------------------------

def best(logits, scores, k, finished=None, pad=0):
    """-> token, parent, score of each request, from float64."""
    b, w, v = logits.shape
    z = logits.astype(np.float64)
    z[np.isnan(z)] = -np.inf
    tok, par, sc = np.full((b, k), pad), np.zeros((b, k), int), np.full((b, k), -np.inf)
    for i in range(b):
        cand = []
        for j in range(w):
            if finished is not None and finished[i, j]:
                cand.append((np.array([float(scores[i, j])]), np.array([j * v + pad])))
                continue
            m = z[i, j].max()
            if not np.isfinite(m):
                continue
            lse = m + np.log(np.exp(z[i, j] - m).sum())
            cand.append((float(scores[i, j]) + (z[i, j] - lse), j * v + np.arange(v)))
        if not cand:
            continue
        s, at = np.concatenate([c[0] for c in cand]), np.concatenate([c[1] for c in cand])
        s[np.isnan(s)] = -np.inf
        order = np.lexsort((at, -s))[:k]
        order = order[s[order] > -np.inf]
        n = len(order)
        tok[i, :n], par[i, :n], sc[i, :n] = at[order] % v, at[order] // v, s[order]
    return tok, par, sc


def select(logits, scores, k, finished=None, pad=0, **kw):
    import torch
    from paper_2609_07966_amd import decoding
    as_dev = lambda x: x if isinstance(x, torch.Tensor) else dev(x)
    got = decoding.beam_select(as_dev(logits), dev(scores), k, finished=None if finished is None else dev(finished),
                               pad_token=pad, **kw)
    return [x.cpu().numpy() for x in got]


def agree(got, want):
    assert np.array_equal(got[0], want[0])
    assert np.array_equal(got[1], want[1])
    fine = np.isfinite(want[2])
    assert np.array_equal(np.isfinite(got[2]), fine)
    # the score's own rounding to float32, and float32 exponentials: relative 2^-22 each (argument rounded
    # to 2^-24 of at most 2^5, result to one unit), which moves the logarithm by as much
    assert np.all(np.abs(got[2][fine] - want[2][fine]) <= 2.0 ** -24 * np.abs(want[2][fine]) + 2.0 ** -18)


def live_scores(rng, b, w):
    return (-rng.random((b, w)) * 5).astype(np.float32)


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("b,w,v,k", [(1, 1, 1, 1), (1, 1, 5, 5), (2, 3, 7, 7), (3, 4, 1000, 8), (1, 4, 32001, 4), (5, 32, 4097, 64),
                                     (2, 8, 16385, 16), (40, 7, 20011, 14), (1, 2, 70001, 64)])
def test_beam_select(b, w, v, k, dtype):
    rng = np.random.default_rng(v + k)
    logits = (rng.standard_normal((b, w, v)) * 3).astype(dtype)
    scores = live_scores(rng, b, w)
    agree(select(logits, scores, k), best(logits, scores, k))


@pytest.mark.parametrize("k", [1, 5, 64])
@pytest.mark.parametrize("kind", ["constant", "two values", "ascending", "descending", "one block"])
def test_beam_ties_and_orders(kind, k):
    v = 40000
    rng = np.random.default_rng(4)
    row = {"constant": np.zeros(v), "two values": (np.arange(v) % 3 == 1) * 1.0, "ascending": np.linspace(-9, 9, v),
           "descending": np.linspace(9, -9, v), "one block": np.where((np.arange(v) >= 9000) & (np.arange(v) < 9300), 5.0, 0.0)}[kind]
    logits = np.broadcast_to(row.astype(np.float32), (2, 3, v)).copy()
    scores = np.array([[0.0, 0.0, 0.0], [-1.0, -0.5, -0.5]], np.float32)  # equal beams: ties go across them
    agree(select(logits, scores, k), best(logits, scores, k))
    half = (np.round(rng.standard_normal((1, 2, v)) * 4) / 4).astype(np.float16)  # many equal values
    agree(select(half, scores[:1, :2], k), best(half, scores[:1, :2], k))


def test_beam_dead_finished_and_banned():
    rng = np.random.default_rng(5)
    b, w, v = 6, 4, 3001
    logits = rng.standard_normal((b, w, v)).astype(np.float32)
    scores = live_scores(rng, b, w)
    finished = np.zeros((b, w), np.uint8)
    scores[0, 1:] = -np.inf                        # a first step: one live beam
    finished[1] = [1, 0, 1, 1]
    finished[2] = 1                                # nothing left to continue
    logits[3, :, 5:] = -np.inf                     # five tokens allowed
    logits[3, 2] = -np.inf                         # a beam with none
    logits[4, 1, ::2] = np.nan
    logits[4, 0] = np.nan
    scores[5] = [np.nan, -np.inf, -1.0, -2.0]
    logits[5, 2, 7:] = -np.inf
    logits[5, 3, 1:] = -np.inf
    for k in (1, 4, 8, 40):
        agree(select(logits, scores, k, finished, pad=17), best(logits, scores, k, finished, pad=17))


def test_beam_strides():
    import torch
    rng = np.random.default_rng(6)
    for dtype in (np.float32, np.float16):
        wide = (rng.standard_normal((12, 5003)) * 2).astype(dtype)
        view = torch.as_strided(dev(wide), (3, 4, 4998), (4 * 5003, 5003, 1), 1)
        logits = wide[:, 1:4999].reshape(3, 4, 4998)
        scores = live_scores(rng, 3, 4)
        agree(select(view, scores, 8), best(logits, scores, 8))


def test_beam_close_scores():
    """Two beams' continuations closer than float32 scores tell apart keep their order in 64 bits."""
    v = 1000
    logits = np.full((1, 2, v), -20.0, np.float32)
    logits[0, :, 3] = 1.0
    lse = 1.0 + np.log1p((v - 1) * np.exp(-21.0))
    scores = np.array([[-100.0, np.nextafter(np.float32(-100.0), np.float32(0))]], np.float32)
    logits[0, 1, 3] = np.float32(1.0)
    got = select(logits, scores, 2)
    assert got[1].tolist() == [[1, 0]] and got[0].tolist() == [[3, 3]]
    assert np.allclose(got[2], scores[:, ::-1] + (1.0 - lse), rtol=2.0 ** -23)


def test_beam_replayed():
    import torch
    from paper_2609_07966_amd import decoding
    rng = np.random.default_rng(7)
    b, w, v, k = 3, 4, 33001, 8
    inputs = [((rng.standard_normal((b, w, v)) * 3).astype(np.float32), live_scores(rng, b, w)) for _ in range(4)]
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        logits, scores = dev(inputs[0][0]), dev(inputs[0][1])
        ws = decoding.beam_workspace(b, w, v, k)
        decoding.beam_select(logits, scores, k, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = decoding.beam_select(logits, scores, k, workspace=ws)
    for x, s in inputs:
        logits.copy_(dev(x))
        scores.copy_(dev(s))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        agree([o.cpu().numpy() for o in out], best(x, s, k))


def test_beam_refusals():
    import torch
    from paper_2609_07966_amd import _lib, decoding
    x, s = torch.zeros((2, 3, 50), device="cuda"), torch.zeros((2, 3), device="cuda")
    for bad in (dict(logits=x.double()), dict(logits=x[..., ::2]), dict(scores=s.half()), dict(scores=s[:1]),
                dict(logits=x.transpose(0, 1)[:, :2]), dict(finished=torch.zeros((2, 3), device="cuda")), dict(scores=s.cpu())):
        with pytest.raises(ValueError):
            decoding.beam_select(**{**dict(logits=x, scores=s, n_select=3), **bad})
    for k, pad in ((0, 0), (51, 0), (65, 0), (3, -1), (3, 50)):
        with pytest.raises(_lib.MkvError) as e:
            decoding.beam_select(x, s, k, pad_token=pad)
        assert e.value.status == 1
    with pytest.raises(_lib.MkvError) as e:
        decoding.beam_select(x, s, 3, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 2
    assert decoding.beam_select(x[:0], s[:0], 3)[0].shape == (0, 3)


@pytest.mark.parametrize("dtype", [np.float32, np.float16])
@pytest.mark.parametrize("w,v,k", [(4, 40000, 8), (3, 1000, 64), (1, 20000, 2), (32, 9000, 64)])
def test_beam_ties_of_scores_whose_logits_differ(w, v, k, dtype):
    """Scores so far from 0 that adding a logit's log-probability changes nothing, as where dead beams are
    given the lowest finite score: continuations tie though their logits do not, and the lower index goes
    first, past what the largest logits would be."""
    rng = np.random.default_rng(8)
    logits = (rng.standard_normal((4, w, v)) * 3).astype(dtype)
    logits[2, :, ::3] = -np.inf
    logits[3, :, :v - k // 2 - 1] = -np.inf
    scores = np.full((4, w), np.finfo(np.float32).min, np.float32)
    scores[1] = -1e30
    scores[1, w // 2] = -2.0                   # one live beam
    finished = np.zeros((4, w), np.uint8)
    if w > 1:
        scores[0, 0] = -3.0                    # finished: one continuation, then the ties of the others
        finished[0, 0] = 1
        finished[1, w - 1] = 1
        finished[2, 1] = 1                     # a tie among the ties
    for f in (None, finished):
        agree(select(logits, scores, k, f, pad=7), best(logits, scores, k, f, pad=7))


def test_beam_ties_of_sums():
    """Logits too small to change their beam's score in 64 bits."""
    rng = np.random.default_rng(9)
    logits = (rng.random((2, 3, 30000)) * 1e-19).astype(np.float32)
    logits[1, :, 20000:] = 2.5                  # some above them
    logits[1, :, 20004:] = -1.0
    scores = np.array([[-2.0, -2.0, -2.5], [-1.0, -1.0, -1.0]], np.float32)
    agree(select(logits, scores, 12), best(logits, scores, 12))
