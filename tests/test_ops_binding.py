"""The binding of the operators around a cache without a GPU."""
import subprocess
import sys

NO_CUDA = """
import torch
for n in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, n)
import paper_2604_15750_b200 as dc
k = torch.zeros((1, 1, 1, 64, 8))
try:
    dc.cache_write(dc.KvCache(k, k.transpose(3, 4).contiguous()), k[:, :, :, :3].transpose(2, 3), k[:, :, :, :3].transpose(2, 3), [0])
except RuntimeError as e:
    assert "no CPU path" in str(e)
else:
    raise SystemExit("not refused")
"""


def test_the_package_comes_in_where_torch_has_no_cuda():
    r = subprocess.run([sys.executable, "-c", NO_CUDA], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
