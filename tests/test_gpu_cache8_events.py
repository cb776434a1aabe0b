"""The timing hook of the decode calls (debug_kernel_events) around those over the 8-bit cache."""
import pytest

from paper_2607_07740_amd import api
from parity_util import say
from test_gpu_cache8 import ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("bifocal", [True, False])
def test_events_are_recorded_around_the_decode_kernel(listed, bifocal):
    cache, lens = api.cache8_alloc(2, 4096, 2), ints([4096, 100])
    q = torch.randn((2, 8, 128), device="cuda").to(torch.bfloat16)
    lists = torch.arange(64, dtype=torch.int32, device="cuda").repeat(2, 2, 1)
    kw = dict(w_pretrained=1000, w_local=100, bifocal=bifocal, workspace=api.decode8_workspace(8, 2))

    def call():
        return api.decode8_blocks(q, cache, lens, lists, **kw) if listed else api.decode8(
            q, cache, lens, **kw)
    want = call()
    before, start, stop, after = (torch.cuda.Event(enable_timing=True) for _ in range(4))
    api.debug_kernel_events(1, start, stop)
    try:
        say("events listed=%s bifocal=%s" % (listed, bifocal))
        torch.cuda.synchronize()
        before.record()
        got = call()
    finally:
        api.debug_kernel_events(1)
    after.record()
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    times = [before.elapsed_time(e) for e in (start, stop, after)]
    assert 0 <= times[0] < times[1] <= times[2], times
    # the hook is cleared: a further call records nothing
    call()
    torch.cuda.synchronize()
    assert before.elapsed_time(stop) == times[1]
