"""Memory of packed weights where they are packed and used on other streams than the current one."""

import pytest
import torch

from tests import clear_util as U
from tests.test_gpu_clear import lib  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def pool_of(t):
    """The stream whose pool a tensor's memory comes from."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]
    raise AssertionError("not from the allocator")


@pytest.mark.parametrize("raw", [False, True])
def test_packed_weights_come_from_the_pool_of_their_stream(lib, raw):
    weight = U.int8(1, 300, 700).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    w = lib.pack_weights(weight, stream=side.cuda_stream if raw else side)
    assert pool_of(w.data) == side.cuda_stream
    assert torch.cuda.current_stream() != side
    assert pool_of(lib.pack_weights(weight).data) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(side):
        assert pool_of(lib.pack_weights(weight).data) == side.cuda_stream
    side.synchronize()
    assert torch.equal(w.data, lib.pack_weights(weight).data)


def test_packed_weights_stay_while_another_stream_uses_them(lib):
    weight, q = U.int8(1, 4000, 4000).cuda(), U.int8(2, 5, 4000).cuda()
    scale, w_scale = torch.ones(5, device="cuda"), torch.ones(4000, device="cuda")
    out = torch.empty((5, 4000), device="cuda")
    side = torch.cuda.Stream()
    w = lib.pack_weights(weight)
    at, size = w.data.data_ptr(), w.data.numel()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)      # about 0.1 s
    for _ in range(2):
        lib.linear(q, scale, w, w_scale, out, stream=side)
    del w
    other = torch.empty(size, dtype=torch.int8, device="cuda")
    assert other.data_ptr() != at           # still in use on the side stream
    other.zero_()
    lib.sync_status(side)
    want = (q.cpu().double() @ weight.cpu().double().T).float()
    assert torch.equal(out.cpu(), want)
