"""Pools whose bitmaps come near the shared memory that a kernel may have without being asked for more: a fresh process for each size, as
a larger pool that was used before on the device would hide what a smaller one lacks."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys
import torch
from paper_2505_21036_b200 import api
P = int(sys.argv[1])
ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
c = api.KVCache.empty(2, 1, 64, P, 4, "cuda")
status, live = ints([0]), ints([0])
last = list(range(P - 1, P - 4, -1))                  # the first sequence lies in the pool's last pages
c.page_table[0, :3] = ints(last)
c.seq_len[0] = 3 * 128
c.k_sum[P - 3:] = torch.tensor([3.0, 2.0, 1.0], device="cuda")[:, None, None]
if sys.argv[2] == "append":
    x = torch.linspace(-448, 448, 130 * 64, device="cuda").to(torch.bfloat16).view(1, 1, 130, 64).expand(2, 1, 130, 64).contiguous()
    api.rf_cache_append(c, x, x, ints([0, 130]), status)
    torch.cuda.synchronize()
    assert int(status) == 0 and c.seq_len.tolist() == [384, 130] and c.page_table[1, :2].tolist() == [0, 1] and c.page_table[0, :3].tolist() == last
    want = x[0, 0].float().to(torch.float8_e4m3fn).float()
    for t in (c.k, c.v):
        assert torch.equal(torch.cat([t[0, 0].float(), t[1, 0, :2].float()]) * torch.cat([c.k_scale[0, 0].expand(128), c.k_scale[1, 0].expand(2)])[:, None], want)
else:
    api.rf_cache_compact(c, live, status)
    torch.cuda.synchronize()
    assert int(status) == 0 and int(live) == 3 and c.page_table[0, :3].tolist() == [2, 1, 0]
    assert c.k_sum[:3, 0, 0].tolist() == [3.0, 2.0, 1.0]
print("fine")
"""


@pytest.mark.parametrize("pages,what", [(146_880, "append"), (147_000, "append"), (190_000, "append"), (196_608, "append"), (196_609, "append"),
                                        (359_000, "compact"), (370_000, "compact"), (393_216, "compact"), (393_250, "compact")])
def test_the_first_call_on_a_pool(pages, what):
    r = subprocess.run([sys.executable, "-c", CHILD, str(pages), what], capture_output=True, text=True, cwd=ROOT, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout[-1000:] + r.stderr[-2000:]
