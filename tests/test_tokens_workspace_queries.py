"""A gradient's workspace query gives what its call takes, for every number of rows: a workspace of that many bytes is enough, and
one for more rows serves fewer.  The calls run in a process that sees no GPU, so that one that is not refused ends at its first
launch; the pointers are never followed."""
import os
import subprocess
import sys

import paper_2601_06562_amd.binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS = (*range(1, 131), 255, 256, 257, 600, 8191, 8193)
HEADS = ((512, 1), (512, 255), (512, 256), (512, 257), (512, 5000), (64, 5), (1032, 32003), (4096, 126464))
SMALL = b.MOSAIC_ERR_WORKSPACE_TOO_SMALL

CALLS = f"""
import sys
sys.path[:0] = [{ROOT!r}, {os.path.join(ROOT, "tests")!r}]
import torch
assert torch.cuda.device_count() == 0
from paper_2601_06562_amd import binding as b
from test_tokens_host_api import logprobs_backward
for d, V in {HEADS}:
    for rows in {ROWS}:
        for budget in (0, 1, 1 << 20):
            need = b.mosaic_masked_logprobs_backward_workspace_bytes(rows, d, V, budget)
            for dw in (dict(dw_type=0), dict(dw_type=1), dict(dw=0)):
                sizes = dict(T=9000, d=d, V=V, max_rows=rows, ld_h=d, ld_w=d, ld_dx=d, ld_dw=d, **dw)
                if need <= 0 or logprobs_backward(bytes=need, **sizes) == {SMALL} or logprobs_backward(bytes=0, **sizes) != {SMALL}:
                    print("refused", rows, d, V, budget, dw)
print("asked")
"""


def test_a_gradient_takes_the_workspace_that_its_query_gives():
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")
    out = subprocess.run([sys.executable, "-c", CALLS], env=env, check=True, stdout=subprocess.PIPE, text=True).stdout
    assert out.split() == ["asked"], out[:2000]


def test_a_smallest_workspace_serves_fewer_rows():
    for d, V in HEADS:
        need = [b.mosaic_masked_logprobs_backward_workspace_bytes(n, d, V, 1) for n in ROWS]
        assert need == sorted(need), (d, V)
