"""The cache operators at the ends of what they take."""
from __future__ import annotations

import pytest
import torch

from oracle import cacheops as oracle
from paper_2608_28099_amd import binding, ops
from tests.test_gpu_ops import rotation_error

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()
    return torch.device("cuda:0")


@pytest.mark.parametrize("layout,dim,n", [("half", 64, (1 << 24) + 5), ("half", 34, (1 << 24) + 5),
                                          ("interleaved", 64, (1 << 26) - 1), ("half", 64, (1 << 26) - 1)])
def test_rotary_of_the_most_rows(dev, layout, dim, n):
    """From 2^24 rows on a launch of one dimension is full (four rows a workgroup: 2^26); in place, against
    calls of fewer rows and, at the end, the definition."""
    rot = ops.make_rotary(64, rotary_dim=dim, layout=layout)
    gen = torch.Generator(device=dev).manual_seed(dim)
    x = torch.randn((n, 1, 64), generator=gen, device=dev, dtype=torch.bfloat16)
    pos = torch.randint(-1, 5000, (n,), generator=gen, device=dev, dtype=torch.int32)
    last, last_pos = x[-300:].cpu(), pos[-300:].cpu()
    ref = x.clone()
    step = 1 << 22
    for i in range(0, n, step):
        ops.rotary(rot, pos[i:i + step], ref[i:i + step], out=ref[i:i + step])
    assert ops.rotary(rot, pos, x, out=x).data_ptr() == x.data_ptr()
    assert torch.equal(x, ref)
    theta, scale = oracle.frequencies(dim)
    live = last_pos >= 0
    want = oracle.rotate(last, last_pos, theta, scale, layout)
    got = x[-300:].cpu()
    assert rotation_error(got[live], last[live], want[live], theta, scale, layout, last_pos[live]) <= 1
    assert torch.equal(got[~live], last[~live])
