"""Paged 8-bit caches on streams other than the current one."""
import pytest
import torch

import test_gpu_pages as T
from paper_2601_20357_b200 import binding as TB

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("current_is_busy", ["default", "side"])
@pytest.mark.parametrize("own_stream", [True, False])
def test_errors_of_first_calls_outlive_the_making_of_the_object(own_stream, current_is_busy):
    """The current stream is busy while an object whose calls run on another one is made and used: what its first call records stays."""
    c = T.make([100], L=1, Hkv=2, ps=64, hd=64)
    given = {x: torch.from_numpy(c[x].copy()).to(T.DEV) for x in T.NAMES}
    bad, z = T.ints([77]), T.ints([0])
    st = torch.cuda.Stream() if own_stream else None
    busy = torch.cuda.Stream() if current_is_busy == "side" else torch.cuda.default_stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(busy):
        torch.cuda._sleep(200_000_000)
        p = TB.Pages(**given, stream=st)
    p.fork(bad, z, z, z)
    torch.cuda.synchronize()
    assert p.last_error() == TB.ERR_INVALID_ARG
    assert p.last_error() == 0


def test_objects_are_made_on_the_device_they_are_of():
    """(one device here: the current stream comes back as it was)"""
    st, c = torch.cuda.Stream(), T.make([100], L=1, Hkv=2, ps=64, hd=64)
    with torch.cuda.stream(st):
        T.to_gpu(c)
        assert torch.cuda.current_stream() == st
        T.to_gpu(c, stream=torch.cuda.Stream())
        assert torch.cuda.current_stream() == st
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
