"""A layer with norm, 8-bit checkpoints and an output layer on the checking build of the library (-DGCNSA_DEBUG), which checks the
places that counted rows are gathered to and the rows that their gradients go to: the same bits as the regular build (this
process; the checking one is a child, as a process loads one library), and nothing recorded."""
import hashlib
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
for path in (os.path.dirname(HERE), HERE):
    if path not in sys.path:
        sys.path.insert(0, path)

pytestmark = pytest.mark.gpu


def scenario():
    import torch
    from paper_2012_04930_b200 import gcnsa
    from test_gpu_norm_head import _ce_run, _problem, _rand, _step, _step_buffers
    out = {}
    for c in (44, 1000):
        torch.manual_seed(c)   # (the labels; the rest has seeds of its own)
        args, _ = _problem(c)
        bufs = _step_buffers(*args[0].shape, args[4].shape[1], c)
        _step(*args, bufs)
        out["step", c] = [bufs[k] for k in ("loss", "h", "dwo", "dbo", "dgamma", "dbeta", "dw", "dt")]
    for n, d, c in ((1, 5, 300), (3001, 33, 129), (5000, 40, 1500)):
        h, w, y = _rand(n, n, d), _rand(d, d, c) / 8, torch.arange(n, device="cuda", dtype=torch.int32) % c
        for share in (0.0, 0.03, 0.6, 1.0):
            mask = (torch.rand(n, generator=torch.Generator().manual_seed(n)) < share).to(torch.uint8).cuda()
            got = _ce_run(h, w, None, y, mask, int(mask.sum()), padded=share < 0.5)
            out["ce", n, share] = list(got.values())
    torch.cuda.synchronize()
    digests = {str(k): hashlib.sha256(b"".join(t.cpu().contiguous().numpy().tobytes() for t in v)).hexdigest() for k, v in out.items()}
    return {"digests": digests, "debug_status": list(gcnsa.debug_status()), "tc_status": gcnsa.tc_status()}


def test_checking_build_gives_the_same_bits_and_records_nothing():
    from paper_2012_04930_b200 import build
    build.build()
    child = subprocess.run([sys.executable, os.path.abspath(__file__), "--child", build.build(debug=True)], capture_output=True, text=True, timeout=900)
    assert child.returncode == 0, child.stderr[-2000:]
    got, want = json.loads(child.stdout.strip().splitlines()[-1]), scenario()
    assert got["debug_status"] == [True, 0, 0], "the checking build recorded a violation (code, value)"
    assert want["debug_status"] == [False, 0, 0] and got["tc_status"] == want["tc_status"] == 0
    assert got["digests"] == want["digests"]


if __name__ == "__main__":
    if len(sys.argv) == 3 and sys.argv[1] == "--child":
        from paper_2012_04930_b200 import gcnsa
        gcnsa.use_library(sys.argv[2])
        print(json.dumps(scenario()))
