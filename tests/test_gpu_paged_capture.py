"""The first calls of a process inside a stream capture: what they set up (kernel attributes, the
module) is set up there, and the graph replays."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

SCRIPT = """
import torch
from paper_2608_08684_gb300 import ripple as lib
dev = "cuda"
B, H, G, d = 3, 2, 4, 128
out = {}
inputs = {}
torch.manual_seed(1)
for name, width in (("short", 4), ("long", 8192)):
    k, v = (torch.randn(16, H, 16, d, device=dev).bfloat16() for _ in range(2))
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    table[:, :4] = torch.arange(12, dtype=torch.int32, device=dev).view(3, 4)
    cache = lib.PagedCache(k, v, table)
    q = torch.randn(B, H * G, d, device=dev).bfloat16()
    new = torch.randn(2, B, H, d, device=dev).bfloat16()
    lens = torch.tensor([50, 1, 64], dtype=torch.int32, device=dev)
    ws = torch.empty(lib.ripple_paged_decode_workspace_bytes(cache, H * G), dtype=torch.uint8,
                     device=dev)
    inputs[name] = (cache, lens, new, q, ws)
logits = {n: torch.randn(*n, device=dev) for n in ((2, 70000), (600, 2000))}
tok = torch.zeros(600, dtype=torch.int32, device=dev)
rope = lib.Rope([0.5 ** i for i in range(d // 2)])


def run():
    for name, (cache, lens, new, q, ws) in inputs.items():
        lib.ripple_paged_append(cache, lens, new[0], new[1], rope=rope)
        lib.ripple_paged_decode_attn(cache, q, lens, out[name], ws)
    for n, x in logits.items():
        lib.ripple_token_logprobs(x, tok[:n[0]], out[n], top_idx=idx[n])


def outputs():
    out.update({name: torch.zeros(B, H * G, d, device=dev) for name in inputs})
    out.update({n: torch.zeros(n[0], device=dev) for n in logits})


idx = {n: torch.zeros(n[0], 3, dtype=torch.int32, device=dev) for n in logits}
outputs()
captured = dict(out)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run()
g.replay()
torch.cuda.synchronize()
outputs()
run()
torch.cuda.synchronize()
for k, x in out.items():
    assert float(x.abs().max()) > 0 and torch.equal(x, captured[k]), k
print("same")
"""


def test_first_calls_inside_a_capture(lib):
    r = subprocess.run([sys.executable, "-c", SCRIPT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "same", r.stderr[-2000:]
