"""The serving operators set no function attribute: the first call of a process may be a captured one, of any of them."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CHILD = """
import sys, json, torch
import paper_2604_12798_amd as vfa
B, Hq, H, d, cap, n, n_q, ns = json.loads(sys.argv[1])
torch.manual_seed(0)
ints = lambda v: torch.full((B,), v, dtype=torch.int32, device="cuda")
x = torch.randn((B, n, Hq + 2 * H, d), device="cuda").to(torch.bfloat16)
a = torch.rand((cap, d), device="cuda")
cache = vfa.kv8_cache(B, H, cap, d)
for t in cache:
    t.fill_(0)
old, new = ints(5), ints(5 + n)
out = [torch.empty((B, h, n, d), dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H)]
back = [torch.empty((B, H, 64, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
q = torch.randn((B, Hq, n_q, d), device="cuda").to(torch.bfloat16)
o, l = torch.empty_like(q), torch.empty((B, Hq, n_q), device="cuda")
ws = torch.empty(vfa.kv8_decode_workspace_bytes(B, Hq, n_q, d, ns), dtype=torch.uint8, device="cuda")
def step():
    vfa.qk_norm_rope_fwd(x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:], cos_sin=a, first_pos=old, out=out)
    vfa.kv8_append(out[1], out[2], cache, old, new)
    vfa.kv8_read(cache, 64, seq_lens=new, out=back)
    vfa.kv8_decode_fwd(q, cache, new, n_splits=ns, workspace=ws, out=o, lse=l)
everything = [*out, *back, o, l]
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    step()
seen = []
for rnd in range(3):
    for t in everything:
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    seen.append([t.clone() for t in everything])
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for s in seen for a, b in zip(s, everything))
assert all(torch.isfinite(t.float()).all() for t in everything)
print("captured", flush=True)
"""


@pytest.mark.parametrize("shape", [(2, 4, 2, 128, 256, 1, 1, 3), (2, 16, 2, 128, 256, 3, 4, 1), (3, 4, 4, 64, 2048, 100, 20, 1)],
                         ids=["step", "drafts_of_32_rows", "d64_one_wide_range"])
def test_first_call_of_a_process_is_captured(shape):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CHILD, json.dumps(shape)], cwd=root, timeout=100, capture_output=True, text=True)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
