"""Calls over the 4-bit cache from two threads at once, whose errors count: a thread that does not end fails the test."""
import threading

import numpy as np
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2511_02043_amd import functional as F

pytestmark = pytest.mark.gpu


def together(jobs):
    """Runs each job in a thread of its own; what they return, or the first error."""
    done = [None] * len(jobs)

    def run(n):
        try:
            done[n] = ("result", jobs[n]())
        except BaseException as e:
            done[n] = ("error", e)

    threads = [threading.Thread(target=run, args=(n,)) for n in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for kind, x in done:
        if kind == "error":
            raise x
    return [x for _, x in done]


def test_an_error_in_a_thread_is_one_of_the_test():
    def refused():
        raise ValueError("refused")
    with pytest.raises(ValueError, match="refused"):
        together([lambda: 1, refused])
    assert together([lambda: 1, lambda: 2]) == [1, 2]


def test_calls_of_two_threads():
    """A decode step and a chunk, each on a stream of its own, twenty times: every result is what the call gives alone."""
    lens, page, r = [900, 333, 1], 16, np.random.default_rng(0)
    jobs, want = [], []
    for D, rows in ((64, 1), (128, 30)):
        caches = [torch.from_numpy(mo.pages_of(r.integers(0, 16, (180, 2, page, D)).astype(np.uint8), r.integers(118, 130, (180, 2, page, D // 32)).astype(np.uint8))).cuda()
                  for _ in range(2)]
        table = torch.from_numpy(r.permutation(180).reshape(3, 60).astype(np.int32)).cuda()
        q, seq = torch.randn(3, 8, rows, D, device="cuda").bfloat16(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        call = F.decode_attention_mx4 if rows == 1 else F.paged_prefill_attention_mx4
        args = (q, *caches, seq, table)
        want.append(call(*args))

        def job(call=call, args=args):
            with torch.cuda.stream(torch.cuda.Stream()):
                got = [call(*args) for _ in range(20)]
                torch.cuda.current_stream().synchronize()
            return got

        jobs.append(job)
    torch.cuda.synchronize()
    for got, w in zip(together(jobs), want):
        assert len(got) == 20 and all(torch.equal(g, w) for g in got)
