"""Products from several host threads at once, each on a stream of its own: a
kernel's first launch sets its limit of LDS, from whichever thread comes first."""
import threading

import pytest
import torch

from paper_2009_13108_amd import niti
from test_gpu_linear import BF16, codes, row_scales

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(1000, 1500, 96), (2000, 1500, 528), (2100, 2100, 1040), (4000, 4000, 128)])
def test_threads(m, n, k):
    a, b = codes(m, k, 1), codes(n, k, 2)
    s_a, s_b = row_scales(m, k, 3), row_scales(n, 1, 4)
    count, errors = 4, []
    outs = [torch.zeros(m, n, dtype=BF16, device="cuda") for _ in range(count)]
    streams = [torch.cuda.Stream() for _ in range(count)]
    torch.cuda.synchronize()
    gate = threading.Barrier(count)

    def work(i):
        try:
            gate.wait(30)
            for _ in range(3):
                niti.linear_fwd(a, b, outs[i], s_a, s_b, stream=streams[i])
        except Exception as e:   # noqa: BLE001 (handed to the test's own thread)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(count)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    torch.cuda.synchronize()
    want = torch.empty_like(outs[0])
    niti.linear_fwd(a, b, want, s_a, s_b)
    assert not errors and all(torch.equal(o, want) for o in outs)
