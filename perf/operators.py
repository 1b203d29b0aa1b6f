"""Performance cases of the operators around a decode step: rotary positions, attention of drafted trees,
acceptance of drafted tokens, beam selection and the reordering of a cache after it.

A case is a dict of plain values.  ``kind`` says what one pass is:

  rope     q and k rows rotated by their positions on one to four axes
  beam     one selection of beams over the vocabulary
  tree     one attention pass of ``nodes`` drafted tokens per sequence over a cache
  reorder  the cache's sequences reordered within groups of ``width`` beams, ``tail`` tokens past a
           prompt of ``prompt``, and one token's attention over the result
  spec     a verification round of sampled drafts: every sequence of a group starts from the group's
           first one, accepts up to ``accept`` drafted tokens, and its next ``nodes`` are attended

``own`` False: plain torch in 32 bits (64 for angles and beam scores).  True: the library's calls.
``lo``, ``hi`` and ``lens`` give prompt lengths (log-uniform in [lo, hi] from the generator seed
``lens``); ``configs`` names compression configurations, dealt to the sequences in turn.
"""
import math
import random

import numpy as np
import torch

own = False

CONFIGS = {
    "FP16": {"method": "fp16"},
    "UQ4": {"method": "uq", "bits": 4, "group": 64},
    "KVQ4": {"method": "kvq", "bits": 4, "outlier_bp": 100},
    "KVQ3": {"method": "kvq", "bits": 3, "outlier_bp": 100},
    "KVQ2": {"method": "kvq", "bits": 2, "outlier_bp": 100},
}
BLOCK = 64  # tokens of a uniform 4-bit key block, channels of a value group
PAD_TOKEN = 2
CHUNK = 64  # nodes of one acceptance when a tail is put into a cache

# Levels of the optimal 4-, 8- and 16-level quantizers of a unit Gaussian (positive half; Max 1960)
_GAUSS = {2: (0.4528, 1.510), 3: (0.2451, 0.7560, 1.344, 2.152),
          4: (0.1284, 0.3881, 0.6568, 0.9424, 1.256, 1.618, 2.069, 2.733)}
_KEY_SPAN, _VALUE_SPAN = 2.576, 2.35


def _rope(name, rows, hq, hkv, d, rot, axes, span, layout="halves", inverse=False):
    return {"name": name, "kind": "rope", "rows": rows, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "axes": axes,
            "span": span, "layout": layout, "inverse": inverse}


def _beam(name, batch, beams, vocab, select, half=False, first=False, finished=0):
    return {"name": name, "kind": "beam", "batch": batch, "beams": beams, "vocab": vocab, "select": select,
            "half": half, "first": first, "finished": finished}


def _tree(name, seqs, hq, hkv, d, lo, hi, configs, nodes, lens=1):
    return {"name": name, "kind": "tree", "seqs": seqs, "hq": hq, "hkv": hkv, "d": d, "lo": lo, "hi": hi,
            "configs": configs, "nodes": nodes, "lens": lens}


def _group(name, kind, groups, width, hq, hkv, d, prompt, configs, tail=0, nodes=1, accept=0):
    return {"name": name, "kind": kind, "groups": groups, "width": width, "hq": hq, "hkv": hkv, "d": d,
            "prompt": prompt, "configs": configs, "tail": tail, "nodes": nodes, "accept": accept}


def listed():
    return [
        # a decode step of 64 sequences far into their contexts: latency
        _rope("rope_step", 64, 32, 8, 128, 128, 1, 100000),
        # a batch of prompts with images and video: time, height and width
        _rope("rope_prompt", 8192, 32, 8, 128, 128, 3, 32768),
        # one request with four beams
        _beam("beam_small", 1, 4, 32001, 4),
        # a batch of requests over a large vocabulary, twice as many candidates as beams
        _beam("beam_large", 16, 8, 128000, 16),
        # a short draft of one conversation on a small model: launches and latency are all there is
        _tree("tree_tiny", 1, 4, 4, 64, 512, 512, "UQ4", 8),
        # a small batch at a medium context, uncompressed and quantized
        _tree("tree_fp16", 8, 32, 8, 128, 4096, 4096, "FP16", 16),
        _tree("tree_kvq", 8, 32, 8, 128, 3000, 6000, "KVQ4,KVQ3,KVQ2", 24),
        # the widest trees over long contexts, each sequence under its own configuration: matrix products
        _tree("tree_wide", 8, 32, 8, 128, 12000, 16384, "FP16,UQ4,KVQ4", 64),
        # beams of a short and of a long generation; the tails move between the beams
        _group("reorder_kvq", "reorder", 4, 4, 32, 8, 128, 1024, "KVQ4", tail=160),
        _group("reorder_fp16", "reorder", 8, 8, 32, 8, 128, 512, "FP16", tail=1000),
        # four sampled drafts of one request, and of a batch under KVQuant
        _group("spec_fp16", "spec", 1, 4, 32, 8, 128, 2048, "FP16", nodes=8, accept=4),
        _group("spec_kvq", "spec", 8, 4, 32, 8, 128, 1500, "KVQ3", nodes=16, accept=6),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((4, 4, 64), (16, 8, 64), (16, 8, 128), (32, 8, 128), (32, 8, 128), (16, 2, 128))


def draw(rng):
    kind = rng.choice(("rope", "beam", "tree", "tree", "reorder", "spec"))
    hq, hkv, d = rng.choice(_HEADS)
    if kind == "rope":
        rot = rng.choice((d, d, d // 2))
        axes = rng.choice((1, 2, 3, 4))
        case = _rope("", _log_uniform(rng, 1, 8192), hq, hkv, d, rot, axes, _log_uniform(rng, 100, 1000000),
                     rng.choice(("halves", "pairs")), rng.random() < 0.3)
    elif kind == "beam":
        beams = rng.choice((1, 2, 3, 4, 5, 8, 16))
        case = _beam("", _log_uniform(rng, 1, 8), beams, _log_uniform(rng, 3000, 128000),
                     min(beams * rng.choice((1, 2)), 32), rng.random() < 0.5, beams > 1 and rng.random() < 0.2,
                     rng.randrange(beams))
    elif kind == "tree":
        seqs = _log_uniform(rng, 1, 8)
        mid = _log_uniform(rng, 64, 8000)
        names = [rng.choice(sorted(CONFIGS)) for _ in range(rng.choice((1, 1, 2, 3)))]
        case = _tree("", seqs, hq, hkv, d, max(1, mid // 2), mid + rng.randrange(mid), ",".join(names),
                     _log_uniform(rng, 1, 64), rng.randrange(1 << 20))
    elif kind == "reorder":
        width = rng.choice((2, 3, 4, 5, 8))
        case = _group("", kind, _log_uniform(rng, 1, 8), width, hq, hkv, d, _log_uniform(rng, 64, 1024),
                      rng.choice(sorted(CONFIGS)), tail=_log_uniform(rng, 16, 800))
    else:
        nodes = _log_uniform(rng, 1, 32)
        case = _group("", kind, _log_uniform(rng, 1, 8), rng.choice((2, 3, 4)), hq, hkv, d,
                      _log_uniform(rng, 64, 2048), rng.choice(("FP16", "KVQ4", "KVQ3", "KVQ2")), nodes=nodes,
                      accept=rng.randrange(1, nodes + 1) if nodes < 8 else rng.randrange(1, 9))
    del case["name"]
    return case


# ---- inputs ----------------------------------------------------------------------------------------

def _lens(case):
    if case["kind"] != "tree":
        return [case["prompt"]] * (case["groups"] * case["width"])
    r = random.Random(case["lens"])
    lo, hi = math.log(case["lo"]), math.log(case["hi"])
    return [int(round(math.exp(r.uniform(lo, hi)))) for _ in range(case["seqs"])]


def _names(case, n):
    names = case["configs"].split(",")
    return [names[s % len(names)] for s in range(n)]


def _books():
    """b = 2, 3, 4: key then value codebook, each entry an fp16 value."""
    books = {}
    for b in (2, 3, 4):
        books[b] = tuple(torch.tensor([-x / span for x in reversed(_GAUSS[b])] + [x / span for x in _GAUSS[b]])
                         .half().float() for span in (_KEY_SPAN, _VALUE_SPAN))
    return books


def _sections(case):
    """Frequency pairs per axis: the first axis takes what an even split leaves."""
    pairs = case["rot"] // 2
    each = pairs // case["axes"]
    return [pairs - each * (case["axes"] - 1)] + [each] * (case["axes"] - 1)


def _rope_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda").half()
    rows, pairs = case["rows"], case["rot"] // 2
    # q and k as one projection leaves them, side by side in a row
    qk = normal(rows, case["hq"] + case["hkv"], case["d"])
    pos = torch.randint(0, case["span"], (case["axes"], rows), generator=g, device="cuda", dtype=torch.int32)
    inv_freq = (10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float()
    return {"qk": qk, "q": qk[:, :case["hq"]], "k": qk[:, case["hq"]:], "pos": pos, "inv_freq": inv_freq,
            "sections": _sections(case)}


def _beam_inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    b, w, v = case["batch"], case["beams"], case["vocab"]
    logits = torch.randn((b, w, v), generator=g, device="cuda") * 2.5
    scores = -torch.rand((b, w), generator=g, device="cuda") * 4.0 - 2.0
    if case["first"]:  # a prompt's first selection: its beams are alike but for the first one's score
        logits = logits[:, :1].expand(b, w, v)
        scores = torch.full((b, w), -math.inf, device="cuda")
        scores[:, 0] = 0.0
    logits = logits.contiguous()
    finished = torch.zeros((b, w), dtype=torch.uint8, device="cuda")
    if case["finished"]:
        finished[:, w - case["finished"]:] = 1
    return {"logits": logits.half() if case["half"] else logits, "scores": scores, "finished": finished}


def _masks(rng, s, n):
    """Random trees: a node's parent is an earlier node or the last cached token (more often near)."""
    masks = np.zeros((s, n), dtype=np.uint64)
    for i in range(s):
        for j in range(n):
            p = rng.randrange(max(-1, j - 6), j) if j else -1
            masks[i, j] = (masks[i, p] if p >= 0 else np.uint64(0)) | (np.uint64(1) << np.uint64(j))
    return torch.from_numpy(masks.view(np.int64)).cuda()


def _cache_inputs(case, seed):
    """Prompt and tail keys and values per sequence, padded to whole blocks [S][Hkv][L][d], the drafted
    nodes' q, k, v and masks, and what the case accepts and reorders.  Keys have per-channel scales
    with two large channels per head."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], case["nodes"]
    lens = _lens(case)
    s = len(lens)
    width = case.get("width", 1)
    tail = case.get("tail", 0)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    sigma = torch.exp(0.5 * normal(s // width, hkv, d))
    big = torch.rand((s // width, hkv, d), generator=g, device="cuda").topk(2, dim=2).indices
    sigma.scatter_(2, big, sigma.gather(2, big) * 8.0)
    sigma = sigma.repeat_interleave(width, 0)  # a group's sequences have one prompt
    room = -(-(max(lens) + tail + case.get("accept", 0)) // BLOCK) * BLOCK
    k = torch.zeros((s, hkv, room, d), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    for i, m in enumerate(lens):
        if i % width == 0:
            k[i, :, :m] = normal(hkv, m, d) * sigma[i, :, None]
            v[i, :, :m] = normal(hkv, m, d)
        else:
            k[i, :, :m], v[i, :, :m] = k[i - 1, :, :m], v[i - 1, :, :m]
        if tail:
            k[i, :, m:m + tail] = normal(hkv, tail, d) * sigma[i, :, None]
            v[i, :, m:m + tail] = normal(hkv, tail, d)
    x = {"lens": lens, "k": k, "v": v, "names": _names(case, s), "tail": tail,
         "q": normal(s, n, hq, d).half(), "kt": (normal(s, n, hkv, d) * sigma[:, None]).half(),
         "vt": normal(s, n, hkv, d).half(), "mask": _masks(rng, s, n)}
    if case["kind"] == "reorder":
        parent = []
        for _ in range(case["groups"]):  # survivors stay where they are, the others follow one of them
            stay = sorted(rng.sample(range(width), rng.randrange(1, width)))
            parent += [w if w in stay else rng.choice(stay) for w in range(width)]
        x["parent"] = torch.tensor(parent, dtype=torch.int32, device="cuda")
    elif case["kind"] == "spec":
        x["parent"] = torch.zeros(s, dtype=torch.int32, device="cuda")
        took = [0 if i % width == 0 else rng.randrange(1, case["accept"] + 1) for i in range(s)]
        path = [sorted(rng.sample(range(n), m)) + [0] * (case["accept"] - m) for m in took]
        x["path"] = torch.tensor(path, dtype=torch.int32, device="cuda")
        x["n_path"] = torch.tensor(took, dtype=torch.int32, device="cuda")
    return x


# ---- a cache in its plain form ---------------------------------------------------------------------
# A part is the sequences of one method: what the cache holds of them, as dense tensors.

def _inverse(top, r):
    """fl32(top / r), 0 where r is 0."""
    return torch.where(r > 0, top / r.double(), 0.0).float()


def _uniform(x):
    """x float32 in groups along the last dimension: 4-bit codes, minimum and step."""
    mn, mx = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    r = mx - mn
    code = torch.round((x - mn) * _inverse(15.0, r)).clamp(0, 15)
    return code.to(torch.uint8), mn, (r.double() / 15.0).float()


def _codes(x, thr, cb):
    """x float32 -> codes (nearest codebook entry of x / thr, [P] codebooks) and outliers (NaN: none)."""
    mids = (cb[:, 1:] + cb[:, :-1]) * 0.5
    xn = (x * _inverse(1.0, thr)).reshape(x.shape[0], -1)
    code = torch.searchsorted(mids, xn.contiguous()).reshape(x.shape).to(torch.uint8)
    return code, torch.where(x.abs() > thr, x, math.nan).half()


def _value_scale(v):
    n_ov = (v.shape[-1] * 100 + 5000) // 10000
    return v.abs().topk(n_ov + 1, dim=-1).values[..., -1:]


def _part(names, lens, k, v, tail):
    p, hkv, room, d = k.shape
    part = {"method": CONFIGS[names[0]]["method"], "count": torch.tensor([n + tail for n in lens], device="cuda")}
    if part["method"] == "fp16":
        part |= {"k": k.clone(), "v": v.clone()}
    elif part["method"] == "uq":
        blocks = k.float().view(p, hkv, room // BLOCK, BLOCK, d).transpose(3, 4).contiguous()
        code, mn, st = _uniform(blocks)
        whole = torch.arange(room, device="cuda") < (part["count"] // BLOCK * BLOCK)[:, None]
        part |= {"kc": code.transpose(3, 4).contiguous(), "kmn": mn.transpose(3, 4).contiguous(),
                 "kst": st.transpose(3, 4).contiguous(),
                 "kr": torch.where(whole[:, None, :, None], math.nan, k.float()).half()}
        part["vc"], part["vmn"], part["vst"] = _uniform(v.float().view(p, hkv, room, d // BLOCK, BLOCK))
    else:
        books = _books()
        pick = lambda side: torch.stack([torch.nn.functional.pad(books[CONFIGS[n]["bits"]][side],
                                                                (0, 16 - (1 << CONFIGS[n]["bits"])), value=math.inf)
                                         for n in names]).cuda()
        part["cbk"], part["cbv"] = pick(0), pick(1)
        n0 = torch.tensor(lens, device="cuda")
        n_o = (n0 * 100 + 5000) // 10000
        prompt = torch.arange(room, device="cuda") < n0[:, None]
        size = torch.where(prompt[:, None, :, None], k.float().abs(), -1.0)
        top = size.topk(int(n_o.max()) + 1, dim=2).values
        part["tau"] = top.gather(2, n_o[:, None, None, None].expand(p, hkv, 1, d))
        part["kc"], part["ko"] = _codes(k.float(), part["tau"], part["cbk"])
        part["vs"] = _value_scale(v.float())
        part["vc"], part["vo"] = _codes(v.float(), part["vs"], part["cbv"])
    return part


def _lookup(cb, code):
    return cb.gather(1, code.view(code.shape[0], -1).long()).view(code.shape)


def _values(part):
    """What a part's cache stands for: keys and values, float32 [P][Hkv][L][d]."""
    if part["method"] == "fp16":
        return part["k"].float(), part["v"].float()
    if part["method"] == "uq":
        kr = part["kr"].float()
        k = (part["kmn"] + part["kc"].float() * part["kst"]).view(kr.shape)
        v = (part["vmn"] + part["vc"].float() * part["vst"]).view(kr.shape)
        return torch.where(torch.isnan(kr), k, kr), v
    ko, vo = part["ko"].float(), part["vo"].float()
    return (torch.where(torch.isnan(ko), _lookup(part["cbk"], part["kc"]) * part["tau"], ko),
            torch.where(torch.isnan(vo), _lookup(part["cbv"], part["vc"]) * part["vs"], vo))


def _attend(part, q, kt, vt, mask):
    """q [P][N][Hq][d], kt, vt [P][N][Hkv][d], mask [P][N] -> [P][N][Hq][d] fp16."""
    k, v = _values(part)
    p, hkv, room, d = k.shape
    n, g = q.shape[1], q.shape[2] // hkv
    rows = q.float().view(p, n, hkv, g, d).transpose(1, 2).reshape(p, hkv, n * g, d) / math.sqrt(d)
    kt, vt = kt.float().transpose(1, 2).contiguous(), vt.float().transpose(1, 2).contiguous()
    s = rows @ k.transpose(2, 3).contiguous()
    dead = torch.arange(room, device="cuda") >= part["count"][:, None]
    s.masked_fill_(dead[:, None, None, :], -math.inf)
    t = (rows @ kt.transpose(2, 3).contiguous()).view(p, hkv, n, g, n)
    seen = (mask[:, :, None] >> torch.arange(n, device="cuda")) & 1
    t = t.masked_fill((seen == 0)[:, None, :, None, :], -math.inf).view(p, hkv, n * g, n)
    m = torch.maximum(s.amax(-1, keepdim=True), t.amax(-1, keepdim=True))
    s, t = torch.exp(s - m), torch.exp(t - m)
    o = (s @ v + t @ vt) / (s.sum(-1, keepdim=True) + t.sum(-1, keepdim=True))
    return o.view(p, hkv, n, g, d).transpose(1, 2).reshape(p, n, hkv * g, d).half()


def _reorder(part, parent, n0):
    """Each sequence of a part takes the tail (and count) of another."""
    part["count"] = part["count"][parent]
    for name, x in part.items():
        if name in ("k", "v", "kr", "kc", "ko", "vc", "vo", "vs", "vmn", "vst", "kmn", "kst"):
            at = n0 // BLOCK if name in ("kmn", "kst") or (name == "kc" and part["method"] == "uq") else n0
            x[:, :, at:] = x[:, :, at:][parent]


def _accept(part, kt, vt, path, n_path):
    """The accepted nodes' keys and values enter the cache behind each sequence's tokens."""
    p, m = path.shape
    seq = torch.arange(p, device="cuda")[:, None].expand(p, m)
    took = torch.arange(m, device="cuda") < n_path[:, None]
    k, v = (x[seq, path.long()].float() for x in (kt, vt))  # [P][M][Hkv][d]
    at = (part["count"][:, None] + torch.arange(m, device="cuda"))[took]
    seq = seq[took]
    if part["method"] == "fp16":
        part["k"][seq, :, at], part["v"][seq, :, at] = k[took].half(), v[took].half()
    else:
        code, out = _codes(k.transpose(1, 2), part["tau"], part["cbk"])
        for name, x in (("kc", code), ("ko", out)):
            part[name][seq, :, at] = x.transpose(1, 2)[took]
        scale = _value_scale(v)
        code, out = _codes(v, scale, part["cbv"])
        for name, x in (("vc", code), ("vo", out), ("vs", scale)):
            part[name][seq, :, at] = x[took]
    part["count"] = part["count"] + n_path


# ---- prepare and run -------------------------------------------------------------------------------

def _library_cache(case, x):
    """The library's cache after the prompts and tails of x."""
    from paper_2609_07966_amd.cache import KVCache
    s, lens = len(x["lens"]), x["lens"]
    flat = [float(y) for b in (2, 3, 4) for cb in _books()[b] for y in cb]
    cache = KVCache((s, case["hq"], case["hkv"], case["d"], x["tail"] + case.get("accept", 0)),
                    [dict(CONFIGS[n]) for n in x["names"]], lens, codebooks=flat)
    rows = lambda t: torch.cat([t[i, :, :m].transpose(0, 1) for i, m in enumerate(lens)]).contiguous()
    cache.append_prompt(rows(x["k"]), rows(x["v"]))
    for a in range(0, x["tail"], CHUNK):
        n = min(CHUNK, x["tail"] - a)
        some = lambda t: t[:, :, lens[0] + a:lens[0] + a + n].transpose(1, 2).contiguous()
        path = torch.arange(n, dtype=torch.int32, device="cuda").expand(s, n).contiguous()
        cache.tree_accept(some(x["k"]), some(x["v"]), path, torch.full((s,), n, dtype=torch.int32, device="cuda"))
    return cache


def prepare(case, seed):
    if case["kind"] == "rope":
        return {"case": case, "x": _rope_inputs(case, seed)}
    if case["kind"] == "beam":
        return {"case": case, "x": _beam_inputs(case, seed)}
    x = _cache_inputs(case, seed)
    state = {"case": case, "x": x, "out": torch.empty_like(x["q"])}
    if own:
        state["cache"] = _library_cache(case, x)
    else:
        by_method = {}
        for i, name in enumerate(x["names"]):
            by_method.setdefault(CONFIGS[name]["method"], []).append(i)
        state["parts"] = [(torch.tensor(at, device="cuda"),
                           _part([x["names"][i] for i in at], [x["lens"][i] for i in at], x["k"][at], x["v"][at], x["tail"]))
                          for at in by_method.values()]
        if "parent" in x:
            first = torch.arange(len(x["lens"]), device="cuda") // case["width"] * case["width"]
            state["from"] = first + x["parent"].long()
    del x["k"], x["v"]
    torch.cuda.synchronize()
    return state


def _run_own(state):
    case, x = state["case"], state["x"]
    if case["kind"] in ("rope", "beam"):
        from paper_2609_07966_amd import decoding
        if case["kind"] == "rope":
            return decoding.rope([x["q"], x["k"]], x["pos"], x["inv_freq"], sections=x["sections"],
                                 layout=case["layout"], inverse=case["inverse"])
        return decoding.beam_select(x["logits"], x["scores"], case["select"], finished=x["finished"],
                                    pad_token=PAD_TOKEN)
    cache = state["cache"]
    if "parent" in x:
        cache.reorder(x["parent"], case["width"])
    if "path" in x:
        cache.tree_accept(x["kt"], x["vt"], x["path"], x["n_path"])
    return cache.tree_attention(x["q"], x["kt"], x["vt"], x["mask"], out=state["out"])


def _run_rope(case, x):
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"),
                                   torch.tensor(x["sections"], device="cuda"), output_size=case["rot"] // 2)
    angle = x["pos"].double()[axis].T * x["inv_freq"].double()
    if case["inverse"]:
        angle = -angle
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    h, rot = case["rot"] // 2, case["rot"]
    qk = x["qk"].float()
    a, b = (qk[..., :h], qk[..., h:rot]) if case["layout"] == "halves" else (qk[..., 0:rot:2], qk[..., 1:rot:2])
    lo, hi = a * c - b * s, b * c + a * s
    turned = torch.cat([lo, hi], -1) if case["layout"] == "halves" else torch.stack([lo, hi], -1).flatten(-2)
    y = torch.cat([turned, qk[..., rot:]], -1).half()
    return [y[:, :case["hq"]].contiguous(), y[:, case["hq"]:].contiguous()]


def _run_beam(case, x):
    b, w, v = x["logits"].shape
    z = x["logits"].double()
    m = z.amax(-1, keepdim=True)
    score = x["scores"].double()[..., None] + (z - m - torch.exp(z - m).sum(-1, keepdim=True).log())
    done = x["finished"].bool()[..., None]
    pad = torch.arange(v, device="cuda") == PAD_TOKEN
    score = torch.where(done, torch.where(pad, x["scores"].double()[..., None], -math.inf), score).view(b, w * v)
    best, at = score.sort(dim=1, descending=True, stable=True)
    best, at = best[:, :case["select"]], at[:, :case["select"]]
    return (at % v).int(), (at // v).int(), best.float()


def run(state):
    if own:
        return _run_own(state)
    case, x = state["case"], state["x"]
    if case["kind"] == "rope":
        return _run_rope(case, x)
    if case["kind"] == "beam":
        return _run_beam(case, x)
    out = state["out"]
    for at, part in state["parts"]:
        if "from" in state:
            _reorder(part, state["from"], case["prompt"])
        if "path" in x:
            _accept(part, x["kt"], x["vt"], x["path"], x["n_path"])
        out[at] = _attend(part, x["q"][at], x["kt"][at], x["vt"][at], x["mask"][at])
    return out


# ---- the least a pass has to do --------------------------------------------------------------------

def _cached_bytes(c, n, d):
    """Bytes that hold n tokens of a kv head."""
    if c["method"] == "fp16":
        return n * 4 * d
    if c["method"] == "uq":
        full = n // BLOCK * BLOCK
        return full * d // 2 + full // BLOCK * d * 8 + (n - full) * 2 * d + n * (d // 2 + d // BLOCK * 8)
    slots = max(1, (d * c["outlier_bp"] + 5000) // 10000)
    return n * (d * c["bits"] // 4 + 8 + 4 * slots) + 4 * n * d * c["outlier_bp"] // 10000


def work(case):
    hq, hkv, d = case.get("hq"), case.get("hkv"), case.get("d")
    if case["kind"] == "rope":
        values = case["rows"] * (hq + hkv) * d
        return {"bytes": float(4 * values + 4 * case["rows"] * case["axes"] + 2 * case["rot"]), "flops": 3.0 * values}
    if case["kind"] == "beam":
        values = case["batch"] * case["beams"] * case["vocab"]
        return {"bytes": float(values * (2 if case["half"] else 4) + case["batch"] * case["select"] * 12),
                "flops": 4.0 * values}
    lens = _lens(case)
    n, nbytes, flops = case["nodes"], 0.0, 0.0
    for m, name in zip(lens, _names(case, len(lens))):
        c = CONFIGS[name]
        held = m + case.get("tail", 0)
        if case["kind"] == "reorder":  # half the beams of a group, more or less, move their tails
            nbytes += hkv * (_cached_bytes(c, held, d) - _cached_bytes(c, m, d))
        if case["kind"] == "spec":
            nbytes += hkv * (_cached_bytes(c, m + case["accept"], d) - _cached_bytes(c, m, d)) / 2
        nbytes += hkv * (_cached_bytes(c, held, d) + n * 4 * d) + n * hq * d * 4 + 8 * n
        flops += 4.0 * n * hq * (held + n / 2) * d
    return {"bytes": nbytes, "flops": flops}


# ---- the same results in 64 bits -------------------------------------------------------------------

def _exact_rope(case, x):
    rot, h = case["rot"], case["rot"] // 2
    at = np.repeat(np.arange(case["axes"]), x["sections"])
    pos, freq = x["pos"].cpu().numpy().astype(np.float64), x["inv_freq"].cpu().numpy().astype(np.float64)
    turn = torch.from_numpy(np.exp((-1j if case["inverse"] else 1j) * (pos[at].T * freq))).cuda()[:, None]
    y = x["qk"].double()
    first, second = (slice(0, h), slice(h, rot)) if case["layout"] == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return [y[:, :case["hq"]].contiguous(), y[:, case["hq"]:].contiguous()]


def _exact_beam(case, x):
    best = []
    for b in range(case["batch"]):
        found = []
        for w in range(case["beams"]):
            if case["finished"] and w >= case["beams"] - case["finished"]:
                found.append(x["scores"][b, w:w + 1].double())
            else:
                found.append(x["scores"][b, w].double() + torch.log_softmax(x["logits"][b, w].double(), 0))
        found = torch.cat(found)
        top = found.topk(min(case["select"], found.numel())).values
        best.append(torch.nn.functional.pad(top, (0, case["select"] - top.numel()), value=-math.inf))
    return None, None, torch.stack(best)


def _exact_uniform(x):
    """x float64, the groups along dimension 0."""
    lo, hi = x.min(0).values, x.max(0).values
    r = (hi.float() - lo.float())
    inv = torch.where(r > 0, 15.0 / r.double(), 0.0).float()
    code = torch.round(((x.float() - lo.float()) * inv)).clamp(0, 15).double()
    return lo + code * (r.double() / 15.0)


def _exact_codes(x, thr, cb):
    """The nearest codebook entry of x / thr times thr; x itself above thr."""
    inv = torch.where(thr > 0, 1.0 / thr.double(), 0.0).float()
    mids = ((cb[1:] + cb[:-1]) * 0.5).contiguous()
    near = cb.double()[torch.searchsorted(mids, (x.float() * inv).contiguous())] * thr.double()
    return torch.where(x.abs() > thr.double(), x, near)


def _exact_tokens(c, k, v, n0):
    """k, v float64 [n][d] of one kv head -> what the cache stands for after n0 prompt tokens and the rest."""
    n, d = k.shape
    if c["method"] == "uq":
        k = torch.cat([_exact_uniform(k[a:a + 64]) if a + 64 <= n else k[a:a + 64] for a in range(0, n, 64)])
        v = torch.cat([_exact_uniform(v[:, a:a + 64].T).T for a in range(0, d, 64)], 1)
    elif c["method"] == "kvq":
        cbk, cbv = (cb.cuda() for cb in _books()[c["bits"]])
        n_o, n_ov = (n0 * 100 + 5000) // 10000, (d * 100 + 5000) // 10000
        tau = k[:n0].abs().sort(0, descending=True).values[n_o].float()
        k = _exact_codes(k, tau, cbk)
        v = _exact_codes(v, v.abs().sort(1, descending=True).values[:, n_ov:n_ov + 1].float(), cbv)
    return k, v


def exact(case, seed):
    if case["kind"] == "rope":
        return _exact_rope(case, _rope_inputs(case, seed))
    if case["kind"] == "beam":
        return _exact_beam(case, _beam_inputs(case, seed))
    x = _cache_inputs(case, seed)
    hkv, g, d, n = case["hkv"], case["hq"] // case["hkv"], case["d"], case["nodes"]
    out = torch.empty(x["q"].shape, dtype=torch.float64, device="cuda")
    masks = x["mask"].cpu().numpy().view(np.uint64)
    for s, n0 in enumerate(x["lens"]):
        src = s
        if "parent" in x:
            src = s // case["width"] * case["width"] + int(x["parent"][s])
        nodes = x["path"][s, :int(x["n_path"][s])].tolist() if "path" in x else []
        seen = torch.tensor([[bool(int(masks[s, i]) >> j & 1) for j in range(n)] for i in range(n)], device="cuda")
        for h in range(hkv):
            end = n0 + x["tail"]
            k = torch.cat([x["k"][src, h, :end], x["kt"][s, nodes, h]]).double()
            v = torch.cat([x["v"][src, h, :end], x["vt"][s, nodes, h]]).double()
            k, v = _exact_tokens(CONFIGS[x["names"][s]], k, v, n0)
            k, v = torch.cat([k, x["kt"][s, :, h].double()]), torch.cat([v, x["vt"][s, :, h].double()])
            rows = x["q"][s, :, h * g:(h + 1) * g].double()  # [N][g][d]
            logit = (rows.reshape(n * g, d) @ k.T.contiguous() / math.sqrt(d)).view(n, g, -1)
            logit[:, :, -n:].masked_fill_(~seen[:, None], -math.inf)
            out[s, :, h * g:(h + 1) * g] = (torch.softmax(logit, -1).view(n * g, -1) @ v).view(n, g, d)
    return out
