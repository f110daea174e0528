"""Two threads on one stream: each call has the bits that it has alone, also where it leaves partial results to a second launch."""
import threading

import pytest
import torch

from test_prompt_paths_gpu import BF, cases, run

pytestmark = pytest.mark.gpu


def test_two_threads_on_one_stream():
    from paper_2503_14985_amd import binding as lib
    ones, others = cases(lib, 0), cases(lib, 50)
    for name in ("packed, keys split", "prompt, keys split", "prefix, few", "prefix, many", "4 bits, rows, K in parts", "4 bits, tiles, K in parts"):
        both = ones[name], others[name]
        want = [run(c) for c in both]
        outs = [[torch.full(c[2], 7.0, dtype=BF, device="cuda") for _ in range(100)] for c in both]
        torch.cuda.synchronize()
        start, errors = threading.Barrier(2), []

        def calls(c, out):
            try:
                start.wait(30)
                for o in out:
                    c[1](c[0], o, None, None)
            except Exception as e:                                   # a thread's own failure would pass unseen
                errors.append(e)

        threads = [threading.Thread(target=calls, args=x) for x in zip(both, outs)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert not errors, errors
        for w, out in zip(want, outs):
            for o in out:
                assert torch.equal(o.view(torch.int16), w.view(torch.int16)), name
