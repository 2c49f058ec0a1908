"""A process whose first call of an eviction is captured into a graph: what the library does once per device does not disturb the capture."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CODE = r"""
import sys
sys.path[:0] = [%r, %r]
import torch
import paper_2507_09071_amd as bs
from cache_util import Paged
torch.manual_seed(3)
c = Paged("bf16", 1, 8, 16, [9000, 7] * 20, capacity=16384, seed=1)
w = torch.rand((40, 1, c.slots), device="cuda:0")
order = torch.arange(c.slots, dtype=torch.int32, device="cuda:0").expand(40, 1, -1).contiguous()
slots = bs.CacheSlots.of(w, order)
ws = torch.empty(bs.bs_cache_evict_workspace(c.cache, 5000), dtype=torch.uint8, device="cuda:0")
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=side):
    bs.bs_cache_evict(c.cache, c.lens, c.lens, 5000, 4, 16, slots, slots, ws, stream=side.cuda_stream)
best = torch.topk(torch.where((order < 4) | (order > 8999 - 16), 2.0, w)[0, 0, :9000], 5000).indices.sort().values
graph.replay()
torch.cuda.synchronize()
assert c.lens.tolist() == [5000, 7] * 20
assert torch.equal(order[0, 0, :5000].sort().values.long(), best)
print("captured and replayed")
"""


def test_first_call_of_a_process_in_a_capture():
    here = os.path.dirname(os.path.abspath(__file__))
    print("capture", flush=True)
    done = subprocess.run([sys.executable, "-c", CODE % (os.path.dirname(here), here)], capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "captured and replayed" in done.stdout, done.stderr
