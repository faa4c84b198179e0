"""The binding of the operators around a cache without a GPU."""
import subprocess
import sys
import types

import pytest

from paper_2604_15750_b200 import ops

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


def test_a_stream_of_another_device_is_refused():
    """The work would go to a device that the tensors are not on."""
    called = []
    with pytest.raises(ValueError, match="device"):
        ops._call(lambda *a: called.append(a) or 0, 0, types.SimpleNamespace(cuda_stream=0, device_index=1))
    assert not called
