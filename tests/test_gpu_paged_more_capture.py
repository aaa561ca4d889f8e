"""The first calls of a process inside a stream capture, for the calls over 8-bit pages and of
drafted tokens: what they set up is set up there, and the graph replays."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

SCRIPT = """
import torch
from paper_2608_08684_gb300 import ripple as lib
dev = "cuda"
B, n, H, G, d = 3, 4, 2, 4, 128
torch.manual_seed(1)
inputs = {}
for kind in ("bf16", "f32", "q8-bf16", "q8-f32"):
    for width in (4, 8192):
        dt = torch.float32 if kind.endswith("f32") else torch.bfloat16
        table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
        table[:, :4] = torch.arange(12, dtype=torch.int32, device=dev).view(3, 4)
        if kind.startswith("q8"):
            k, v = (torch.randint(0, 120, (16, H, 16, d), dtype=torch.uint8, device=dev) for _ in "kv")
            s = torch.full((2, 16, H, 16), 120, dtype=torch.uint8, device=dev).view(torch.float8_e8m0fnu)
            cache = lib.PagedCache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), table,
                                   k_scales=s[0], v_scales=s[1], dtype=dt)
        else:
            k, v = (torch.randn(16, H, 16, d, device=dev).to(dt) for _ in "kv")
            cache = lib.PagedCache(k, v, table)
        q = torch.randn(B, n, H * G, d, device=dev).to(dt)
        new = torch.randn(2, B, n, H, d, device=dev).to(dt)
        ws = torch.empty(max(lib.ripple_paged_decode_workspace_bytes(cache, H * G),
                             lib.ripple_paged_tree_workspace_bytes(cache, H * G, n)),
                         dtype=torch.uint8, device=dev)
        inputs[kind, width] = (cache, new, q, ws, lib.KeepTables([cache]))
lens = torch.tensor([[50, 4, 64]], dtype=torch.int32, device=dev)
kept = torch.tensor([[0, 2], [1, -1], [2, 3]], dtype=torch.int32, device=dev)
rope = lib.Rope([0.5 ** i for i in range(d // 2)])


def run(out):
    for key, (cache, new, q, ws, keep) in inputs.items():
        tree, dec, lens_out = out[key]
        lib.ripple_paged_append(cache, lens[0], new[0], new[1], rope=rope)
        lib.ripple_paged_tree_attn(cache, q, lens[0], tree, ws)
        lib.ripple_paged_decode_attn(cache, q[:, 0], lens[0], dec, ws)
        lib.ripple_paged_keep_rows(keep, lens, kept, n_tokens=n, lens_out=lens_out)


def outputs():
    return {key: (torch.zeros_like(x[2]), torch.zeros(B, H * G, d, device=dev), torch.zeros_like(lens))
            for key, x in inputs.items()}


captured = outputs()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run(captured)
g.replay()
torch.cuda.synchronize()
again = outputs()
run(again)
torch.cuda.synchronize()
for key in inputs:
    for x, y in zip(captured[key], again[key]):
        assert float(x.abs().max()) > 0 and torch.equal(x, y), key
print("same")
"""


def test_first_calls_inside_a_capture(lib):
    r = subprocess.run([sys.executable, "-c", SCRIPT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
