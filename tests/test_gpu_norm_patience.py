"""The norms' backward pass waits for the rows that it copies into shared memory, and the wait has an end.  When it runs out nothing of what the
call makes may pass for a result: every output is NaN, the sums too, nothing is written elsewhere, and the copies still in flight have landed
before their place is used again.  LML_NORM_PATIENCE is read once per process: a child process with patience 0 waits for no row."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys
sys.path.insert(0, %r); sys.path.insert(0, %r)
import torch
from gpu_util import Guarded
from paper_2608_15241_b200 import binding as b
g = torch.Generator(device="cuda").manual_seed(1)
mk = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
# one row, rows beyond the ring, several groups of warps, two and four vectors per thread, the kernels of the usual call and the others
for T, d in ((1, 64), (300, 264), (1000, 1024), (400, 5120), (700, 8192), (200, 16384)):
    for form in ("bf16", "int8", "e4m3"):
        for gate in ("shared", "rows", "none"):
            for sums in (True, False):
                keep = (lambda t: t) if form == "bf16" else (lambda t: b.checkpoint_store(t, form))
                h, o, dx, dh_new = (mk(T, d) for _ in range(4))
                norm = b.BlockNorm(d, w_post=mk(d), w_pre=mk(d), gate=mk(d) if gate == "shared" else None)
                gates = mk(T, d) if gate == "rows" else None
                out = [Guarded(T * d * 2, fill=0) for _ in range(3)]
                dh, d_o, dg = (x.view(torch.bfloat16, (T, d)) for x in out)
                gs, ws = Guarded(3 * d * 4, fill=0), Guarded(b.lml_block_norm_workspace_bytes(0, T, d), fill=0)
                w = gs.view(torch.float32, (3, d))
                p = lambda t: 0 if t is None else t.data_ptr()
                b.lml_block_norm_backward(0, norm.desc, T, b._as_rows(keep(h), (T, d), "h", 0), b._as_rows(keep(o), (T, d), "o", 0), p(gates), p(dx), p(dh_new),
                                          p(dh), p(d_o), p(w[0]) if sums else 0, p(w[1]) if sums else 0, p(w[2]) if sums and gate == "shared" else 0,
                                          p(dg) if gate == "rows" else 0, p(ws.payload) if sums else 0, ws.nbytes if sums else 0,
                                          torch.cuda.current_stream().cuda_stream)
                torch.cuda.synchronize()
                here = (T, d, form, gate, sums)
                assert all(x.intact() for x in out) and gs.intact() and ws.intact(), here
                assert torch.isnan(dh).all() and torch.isnan(d_o).all(), here
                assert torch.isnan(dg).all() if gate == "rows" else (dg == 0).all(), here
                assert torch.isnan(w[:2]).all() if sums else (w == 0).all(), here
                assert torch.isnan(w[2]).all() if sums and gate == "shared" else (w[2] == 0).all(), here
# parts that are not there: only dx, only dh', no block before
T, d = 500, 520
h, o, dx, dh_new = (mk(T, d) for _ in range(4))
norm = b.BlockNorm(d, w_post=mk(d), w_pre=mk(d))
for args in ((h, o, dx, None), (None, o, None, dh_new), (h, None, dx, dh_new)):
    sums = torch.zeros(d, device="cuda")
    dh, d_o, _ = norm.backward(*args, dw_pre=sums if args[2] is not None else None, dw_post=sums if args[2] is None else None)
    torch.cuda.synchronize()
    assert torch.isnan(dh).all() and (d_o is None or torch.isnan(d_o).all()) and torch.isnan(sums).all()
# the forward pass has no such wait
h_new, x = norm.forward(h, o)
torch.cuda.synchronize()
assert torch.isfinite(h_new.float()).all() and torch.isfinite(x.float()).all()
print("ok")
"""


def test_rows_that_do_not_come_in_time_make_every_result_nan():
    env = dict(os.environ, LML_NORM_PATIENCE="0")
    r = subprocess.run([sys.executable, "-c", CHILD % (ROOT, os.path.join(ROOT, "tests"))], env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout[-2000:] + r.stderr[-2000:]
