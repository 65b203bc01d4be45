"""A kernel's first call of a process is one that is captured: nothing has been loaded, and no limit raised, ahead of it."""
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu

_START = """
import torch
from paper_2311_02382_amd import lss
gen = torch.Generator().manual_seed(3)
normal = lambda *s, dt=torch.bfloat16: torch.randn(s, generator=gen).to(dt).cuda()
i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
scratch = lambda n: torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda")
"""
_SELECT = """
B, K, V, N = {sizes}
logits, scores, ws = normal(B * K, V, dt=torch.{dtype}), normal(B, K, dt=torch.float32), scratch(lss.lss_beam_select_workspace_bytes(B, K, V, N))
made = lambda: (torch.zeros(B, N, device="cuda"), torch.zeros(B, N, dtype=torch.int32, device="cuda"), torch.zeros(B, N, dtype=torch.int32, device="cuda"))
call = lambda a: lss.lss_beam_select(logits, scores, N, scores_out=a[0], parents=a[1], tokens=a[2], workspace=ws)
"""
_TREE = """
new, length = {sizes}
kc, vc, q, table = normal(200, 16, 2, 64), normal(200, 16, 2, 64), normal(new, 8, 64), torch.randperm(200, generator=gen).int().view(1, 200).cuda()
lengths, cu, ws = i32([length]), i32([0, new]), scratch(lss.lss_paged_attn_tree_workspace_bytes(new, 1, 8, 2, 64, 3200))
made = lambda: (torch.zeros(new, 8, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(new, 8, device="cuda"))
call = lambda a: lss.lss_paged_attn_tree(q, kc, vc, table, lengths, cu, out=a[0], lse=a[1], workspace=ws)
"""
_END = """
first, second = made(), made()
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    call(first)
for i in range(3):
    for x in first:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    call(second)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, second)) and any(bool((x != 0).any()) for x in first), i
print("alike")
"""


# beams whose lists take more LDS than a launch has without asking, from the logits themselves and by a launch in front; drafted tokens, few and many
@pytest.mark.parametrize("call", [_SELECT.format(sizes="2, 16, 4000, 64", dtype="float32"), _SELECT.format(sizes="2, 16, 4000, 64", dtype="bfloat16"),
                                  _SELECT.format(sizes="1, 32, 9000, 64", dtype="bfloat16"), _TREE.format(sizes="3, 2000"), _TREE.format(sizes="100, 3000")],
                         ids=["select float", "select", "select wide", "tree", "tree wide"])
def test_first_call_is_captured(call):
    r = subprocess.run([sys.executable, "-c", _START + call + _END], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and r.stdout.strip().endswith("alike"), (r.returncode, r.stdout[-500:], r.stderr[-2000:])
