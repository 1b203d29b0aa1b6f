"""Torch-facing convenience over the C ABI: owns the arena tensor and marshals tensors to pointers.

PyTorch only provides device memory and the stream here; every step of the decode path runs in
libmkv's HIP kernels.
"""
import struct

from . import _lib as L


def _ptr(t):
    return 0 if t is None else int(t.data_ptr())


def raw_stream(device):
    """The current stream of a device as a hipStream_t (torch.cuda.current_stream makes an object first,
    which takes longer than a launch)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def check_tensor(name, t, device, dtype, shape):
    """A call that reads a device buffer by its pointer needs it to be what the kernels take it for."""
    if t.device != device or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {device} "
                         f"(got {t.dtype}, {tuple(t.shape)} on {t.device})")


def check_workspace(t, device):
    """(Its size and alignment are the library's to check.)"""
    import torch
    if t.device != device or t.dtype != torch.uint8 or not t.is_contiguous():
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {device} (got {t.dtype} on {t.device})")


class KVCache:
    """One mixed-configuration KV cache (one attention layer's worth).

    shape: (n_seqs, n_q_heads, n_kv_heads, head_dim, max_new_tokens)
    cfgs:  per-sequence configuration dicts (workloads.configs rows)
    codebooks: flat 56 float32 values (b = 2, 3, 4: key then value codebook), or None

    Every call enqueues on the stream the cache was made with (`stream`, or the one current then).  The prefill
    and decode calls do no more: whoever makes their inputs or reads their outputs on another stream orders
    the two.  tree_attention, tree_accept and reorder, which go with the calls of `decoding` on the current
    stream, are ordered with the current stream where it is another one.  (That is some 27 us of host time a
    call, for two events; none where the cache's stream is the current one.  A captured call needs a cache made
    with a stream of its own: the default stream cannot join a capture.)
    """

    def __init__(self, shape, cfgs, prompt_lens, codebooks=None, device="cuda", stream=None):
        import torch
        self.torch = torch
        self.shape = tuple(int(x) for x in shape)
        self.S, self.Hq, self.Hkv, self.D, self.max_new = self.shape
        self.cfgs = [dict(c) for c in cfgs]
        self.prompt_lens = [int(x) for x in prompt_lens]
        rows = [L.make_config(c) for c in self.cfgs]
        self._tree_bytes = {}  # nodes -> workspace bytes, which the cache's layout settles
        self.nbytes = L.mkv_cache_bytes(self.shape, rows, self.prompt_lens)
        self.arena = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        base = self.arena.data_ptr()
        self.arena_ptr = (base + 255) & ~255
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.arena.device)
        self.h = L.mkv_cache_create(self.shape, rows, self.prompt_lens, codebooks, self.arena_ptr,
                                    self.nbytes, self.stream.cuda_stream)

    def close(self):
        if getattr(self, "h", None):
            L.mkv_cache_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def s(self):
        return self.stream.cuda_stream

    # ---- prefill -----------------------------------------------------------------------------
    def append_prompt(self, k, v):
        """k, v: device fp16 [sum prompt_len][Hkv][D] (sequences in order)."""
        cu = [0]
        for n in self.prompt_lens:
            cu.append(cu[-1] + n)
        L.mkv_append_quantize(self.h, _ptr(k), _ptr(v), cu, self.s)

    def h2o_prefill(self, q_prompt):
        L.mkv_h2o_update_evict(self.h, _ptr(q_prompt), self.s)

    def snap_prefill(self, q_window):
        L.mkv_snap_prefill_evict(self.h, _ptr(q_window), self.s)

    # ---- decode ------------------------------------------------------------------------------
    def append(self, k, v):
        L.mkv_append_quantize(self.h, _ptr(k), _ptr(v), list(range(self.S + 1)), self.s)

    def topk(self, q, pos_out=None):
        L.mkv_topk_select(self.h, _ptr(q), _ptr(pos_out), self.s)

    def attention(self, q, out):
        L.mkv_decode_attention(self.h, _ptr(q), _ptr(out), self.s)

    def evict(self):
        L.mkv_h2o_update_evict(self.h, 0, self.s)

    def step(self, k, v, q, out):
        L.mkv_decode_step(self.h, _ptr(k), _ptr(v), _ptr(q), _ptr(out), self.s)

    # ---- drafted trees (mkv_tree_attention, mkv_tree_accept) ----------------------------------
    def tree_workspace(self, n_nodes):
        """A workspace of tree_attention for n_nodes nodes (torch aligns an allocation to 512 bytes)."""
        if n_nodes not in self._tree_bytes:
            self._tree_bytes[n_nodes] = L.mkv_tree_workspace(self.h, n_nodes)
        return self.torch.empty(self._tree_bytes[n_nodes], dtype=self.torch.uint8, device=self.arena.device)

    def tree_attention(self, q, k, v, mask, out=None, n_valid=None, workspace=None):
        """Attention of drafted nodes over the cache and each other -> out [S][N][Hq][D] fp16.

        q [S][N][Hq][D], k, v [S][N][Hkv][D] fp16; mask [S][N] int64, bit j of a node's word = it
        attends to node j; n_valid: optional int32 [S], the nodes each sequence has (rows of others stay as
        they are in `out`, and undefined without one).  The default workspace is allocated for the call."""
        torch, dev = self.torch, self.arena.device
        n = q.shape[1] if q.dim() == 4 else 0
        check_tensor("q", q, dev, torch.float16, (self.S, n, self.Hq, self.D))
        check_tensor("k", k, dev, torch.float16, (self.S, n, self.Hkv, self.D))
        check_tensor("v", v, dev, torch.float16, (self.S, n, self.Hkv, self.D))
        check_tensor("mask", mask, dev, torch.int64, (self.S, n))
        if n_valid is not None:
            check_tensor("n_valid", n_valid, dev, torch.int32, (self.S,))
        if out is not None:
            check_tensor("out", out, dev, torch.float16, (self.S, n, self.Hq, self.D))
        ws = workspace
        if ws is not None:
            check_workspace(ws, dev)
        # (allocated on the current stream, whose further work comes behind the call)
        if out is None:
            out = torch.empty_like(q)
        if ws is None:
            ws = self.tree_workspace(n)
        self._launch(L.mkv_tree_attention, _ptr(q), _ptr(k), _ptr(v), _ptr(mask), _ptr(n_valid), n, _ptr(out), _ptr(ws),
                     ws.numel())
        return out

    def _launch(self, fn, *args):
        """fn(handle, *args, stream) with the cache's device current.  Where another stream than the cache's is
        current, the call comes behind that stream's work, and its further work behind the call: tensors
        written, read or freed there need no care."""
        device = self.arena.device
        if self.torch.cuda.current_device() != device.index:
            with self.torch.cuda.device(device):
                return self._launch(fn, *args)
        if raw_stream(device) == self.s:
            fn(self.h, *args, self.s)
        else:
            current = self.torch.cuda.current_stream(device)
            self.stream.wait_stream(current)
            try:
                fn(self.h, *args, self.s)
            finally:  # (a stream that has joined a capture has to come back, also from a refused call)
                current.wait_stream(self.stream)

    def tree_accept(self, k, v, path, n_path, counts=None):
        """Append nodes path[s][:n_path[s]] of k, v [S][N][Hkv][D] to each sequence; path [S][M], n_path [S]
        int32; counts: optional int32 [S], receives the tokens each sequence then holds."""
        torch, dev = self.torch, self.arena.device
        n = k.shape[1] if k.dim() == 4 else 0
        m = path.shape[1] if path.dim() == 2 else 0
        check_tensor("k", k, dev, torch.float16, (self.S, n, self.Hkv, self.D))
        check_tensor("v", v, dev, torch.float16, (self.S, n, self.Hkv, self.D))
        check_tensor("path", path, dev, torch.int32, (self.S, m))
        check_tensor("n_path", n_path, dev, torch.int32, (self.S,))
        if counts is not None:
            check_tensor("counts", counts, dev, torch.int32, (self.S,))
        self._launch(L.mkv_tree_accept, _ptr(k), _ptr(v), n, _ptr(path), _ptr(n_path), m, _ptr(counts))

    # ---- beams (mkv_cache_reorder) -------------------------------------------------------------
    def reorder(self, parent, width):
        """Beam w of group g takes the state of beam parent[g * width + w] (int32 [S]) of its group."""
        check_tensor("parent", parent, self.arena.device, self.torch.int32, (self.S,))
        self._launch(L.mkv_cache_reorder, _ptr(parent), width)

    # ---- inspection --------------------------------------------------------------------------
    def export(self, seq, kv_head, what, dtype=None):
        import numpy as np
        raw = L.mkv_export(self.h, seq, kv_head, what)
        if dtype is None:
            dtype = {"codes_k": np.uint8, "codes_v": np.uint8, "scales_k": np.float32, "scales_v": np.float32,
                     "scores": np.float32}.get(what, np.int32)
        return np.frombuffer(raw, dtype=dtype).copy()

    def counts(self, seq, kv_head):
        return struct.unpack("4i", L.mkv_export(self.h, seq, kv_head, "counts"))

    def n_tiles(self):
        """-> (all attention tiles, tiles of uniform 4-bit sequences, tiles of RocketKV sequences)."""
        return L.mkv_attention_tiles(self.h)
