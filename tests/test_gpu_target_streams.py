"""The target-side calls from several threads, each on a stream of its own and without a workspace, give each its answers."""
import threading

import pytest
import torch

from paper_2609_21858_gb300 import pps
from test_gpu_attention import BF, F16, Case, _cuda  # noqa: F401
from test_gpu_chain import _chains

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("named", [False, True])
def test_threads(named):
    jobs = []
    for i in range(6):
        attend = Case([1, 1 + 7 * i, 40], [3000 + 500 * i, 200, 900], 8, 2, 128 if i % 2 else 64, 16, F16 if i % 2 else BF, seed=i)
        chain = _chains([5, i, 0, 3], 20000 + 999 * i, BF, i)
        jobs.append((attend, chain, attend.call(), pps.verify_chain(*chain)))
    torch.cuda.synchronize()
    wrong = []

    def work(attend, chain, out, verified):
        try:
            stream = torch.cuda.Stream()
            kw = dict(stream=stream) if named else {}
            with torch.cuda.stream(stream):
                for _ in range(30):
                    a, b = attend.call(**kw), pps.verify_chain(*chain, **kw)
                    if not torch.equal(a, out) or any(not torch.equal(b[k], verified[k]) for k in verified):
                        wrong.append("differs")
                stream.synchronize()
        except Exception as e:  # a thread's exception would be lost
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
