"""Torch-facing calls of the operators that need no cache: rotary positions and beam selection.

PyTorch provides device memory and the stream; the work runs in libmkv's HIP kernels, on the
current stream of the tensors' device.
"""
import torch

from . import _lib as L
from .cache import check_tensor, check_workspace, raw_stream


def _launch(device, fn, *args):
    """fn(*args, stream) with the device current and its current stream."""
    if torch.cuda.current_device() == device.index:
        fn(*args, raw_stream(device))
    else:
        with torch.cuda.device(device):
            fn(*args, raw_stream(device))


def rope(xs, pos, inv_freq, sections=None, layout="halves", inverse=False, out=None):
    """Rotate the rows of each tensor of xs ([rows][heads][head_dim] fp16: a token's queries, its keys)
    by their positions -> a list of outputs.

    A row's heads are contiguous, the rows at any distance.  pos int32 [axes][rows]; inv_freq float32
    [rotary_dim / 2]; sections: frequency pairs per axis (default: all of the one axis); layout
    "halves" or "pairs"; inverse: turn back (the gradient).  out: tensors to write, which may be xs
    themselves (default: new ones)."""
    dev = xs[0].device
    n_rows, _, d = xs[0].shape
    sections = (inv_freq.numel(),) if sections is None else sections
    pairs = sum(sections)
    check_tensor("pos", pos, dev, torch.int32, (len(sections), n_rows))
    check_tensor("inv_freq", inv_freq, dev, torch.float32, (pairs,))
    if len(sections) > L.ROPE_MAX_AXES:
        raise ValueError(f"at most {L.ROPE_MAX_AXES} axes (got {len(sections)})")
    if n_rows >= 2 ** 31:
        raise ValueError("too many rows")
    if layout not in L.ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(L.ROPE_LAYOUTS)} (got {layout!r})")
    if out is not None and len(out) != len(xs):
        raise ValueError("out has another number of tensors than xs")
    ys, sets = [], []
    for i, x in enumerate(xs):
        shape = x.shape
        if len(shape) != 3 or shape[0] != n_rows or shape[2] != d:
            raise ValueError("xs are [rows][heads][head_dim] and agree in rows and head_dim")
        heads = shape[1]
        x_stride = y_stride = heads * d
        _rows(x, dev, heads, d)
        if n_rows > 1:  # (one row has any stride)
            x_stride = x.stride(0)
        if out is None:
            y = x.new_empty(shape)
        else:
            y = out[i]
            if y.shape != shape:
                raise ValueError("out has the shapes of xs")
            _rows(y, dev, heads, d)
            if n_rows > 1:
                y_stride = y.stride(0)
        ys.append(y)
        sets.append((x.data_ptr(), y.data_ptr(), x_stride, y_stride, heads))
    if n_rows > 0:
        _launch(dev, L.mkv_rope, d, 2 * pairs, sections, layout, inv_freq.data_ptr(), pos.data_ptr(), n_rows, sets, inverse)
    return ys


def _rows(t, dev, heads, d):
    if t.device != dev or t.dtype != torch.float16:
        raise ValueError(f"xs and out must be float16 on {dev}")
    stride = t.stride()
    if stride[2] != 1 or (heads > 1 and stride[1] != d):
        raise ValueError("a row's heads must be contiguous (rows may be any distance apart)")


def beam_workspace(n_batch, n_beams, vocab, n_select, device="cuda"):
    """A workspace of beam_select, for calls that may overlap or be captured."""
    return torch.empty(L.mkv_beam_workspace(n_batch, n_beams, vocab, n_select), dtype=torch.uint8, device=device)


def beam_select(logits, scores, n_select, finished=None, pad_token=0, workspace=None):
    """The n_select best continuations of each request's beams -> (token, parent int32, score float32),
    each [batch][n_select], best first.

    logits [batch][beams][vocab] float32 or float16 (rows may be any distance apart); scores float32
    [batch][beams]; finished: optional uint8 [batch][beams], beams that continue with pad_token alone."""
    dev = logits.device
    b, w, v = logits.shape
    if logits.dtype not in (torch.float32, torch.float16) or logits.stride(2) != 1 or \
            (b > 1 and logits.stride(0) != w * logits.stride(1)):
        raise ValueError("logits must be float32 or float16 with contiguous rows at one distance")
    check_tensor("scores", scores, dev, torch.float32, (b, w))
    if finished is not None:
        check_tensor("finished", finished, dev, torch.uint8, (b, w))
    stride = logits.stride(1) if w > 1 else logits.stride(0) if b > 1 else v
    token = torch.empty((b, n_select), dtype=torch.int32, device=dev)
    parent, score = torch.empty_like(token), scores.new_empty((b, n_select))
    if workspace is not None:
        check_workspace(workspace, dev)
    if b * w >= 2 ** 31:
        raise ValueError("too many rows")
    ws = workspace if workspace is not None else beam_workspace(b, w, v, n_select, dev)
    _launch(dev, L.mkv_beam_select, logits.data_ptr(), L.F16 if logits.dtype == torch.float16 else L.F32, stride, b, w, v,
            scores.data_ptr(), 0 if finished is None else finished.data_ptr(), pad_token, n_select, token.data_ptr(),
            parent.data_ptr(), score.data_ptr(), ws.data_ptr(), ws.numel())
    return token, parent, score
