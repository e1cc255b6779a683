"""Calls of head_logits of different sizes by several host threads at once."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_calls_of_two_sizes_at_once(gls, dtype):
    """The kernel is the same and its shared memory is not: neither thread's call may fail for the other's."""
    g = torch.Generator(device="cuda").manual_seed(1)
    tables = [gls.quantize_table(torch.randn((V, D), generator=g, device="cuda"), group=128) for V, D in ((300, 512), (200, 2560))]
    xs = [torch.randn((n, t.dim), generator=g, device="cuda").to(dtype) for n, t in zip((3, 4), tables)]
    want = [gls.head_logits(x, t) for x, t in zip(xs, tables)]
    failed = []

    def run(i, stream):
        try:
            with torch.cuda.stream(stream):
                for _ in range(3000):
                    got = gls.head_logits(xs[i], tables[i])
                stream.synchronize()
                if not torch.equal(got, want[i]):
                    failed.append("thread %d: other logits" % i)
        except Exception as e:  # noqa: BLE001
            failed.append("thread %d: %r" % (i, e))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i, torch.cuda.Stream())) for i in (0, 1, 0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
