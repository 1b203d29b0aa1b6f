"""The host side of the operators around a decode step (argument checks, workspace plans) built with
AddressSanitizer and UndefinedBehaviorSanitizer on host code only and run on the CPU through a small native
driver (tests/native/decoding_checks.cpp) whose kernel launchers are stubs; and the torch wrappers'
refusals, which come before anything reaches the library."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_decoding_host_code_under_asan_and_ubsan(tmp_path):
    csrc = os.path.join(ROOT, "paper_2609_07966_amd", "csrc")
    exe = str(tmp_path / "decoding_checks")
    cmd = [HIPCC, "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
           "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "decoding.cpp"),
           os.path.join(ROOT, "tests", "native", "decoding_checks.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "ok (0 failures)" in r.stdout


def test_wrapper_refusals():
    torch = pytest.importorskip("torch")
    from paper_2609_07966_amd import decoding
    x = torch.zeros((3, 2, 64), dtype=torch.float16)
    pos, f = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(32)
    for bad in (dict(xs=[x.float()]), dict(xs=[x, x[:2]]), dict(pos=pos.long()), dict(pos=pos[:, :2]), dict(inv_freq=f.double()),
                dict(sections=[31]), dict(sections=[8, 8, 8, 4, 4], pos=torch.zeros((5, 3), dtype=torch.int32)), dict(layout="other"),
                dict(out=[x, x]), dict(xs=[x.transpose(0, 1)]), dict(out=[x[:, :1]]), dict(xs=[x[..., ::2]]), dict(out=[x.double()])):
        with pytest.raises(ValueError):
            decoding.rope(**{**dict(xs=[x], pos=pos, inv_freq=f), **bad})
    z, s = torch.zeros((2, 3, 50)), torch.zeros((2, 3))
    for bad in (dict(logits=z.double()), dict(logits=z[..., ::2]), dict(scores=s.half()), dict(scores=s[:1]),
                dict(logits=z.transpose(0, 1)[:, :2]), dict(finished=torch.zeros((2, 3)))):
        with pytest.raises(ValueError):
            decoding.beam_select(**{**dict(logits=z, scores=s, n_select=3), **bad})
    # a workspace that is not bytes, or not all there, or elsewhere
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for bad in (ws.float(), ws[::2], ws.to("meta")):
        with pytest.raises(ValueError):
            decoding.beam_select(z, s, 3, workspace=bad)
    # more rows than the library counts
    n = 2 ** 31
    wide = torch.empty((n, 1, 2), dtype=torch.float16, device="meta")
    with pytest.raises(ValueError):
        decoding.rope([wide], torch.empty((1, n), dtype=torch.int32, device="meta"), torch.empty(1, device="meta"))
    with pytest.raises(ValueError):
        decoding.beam_select(torch.empty((n, 1, 1), device="meta"), torch.empty((n, 1), device="meta"), 1)
