"""MOE_DEBUG_SYNC=1: every launch of an entry point is followed by a synchronisation, so
that a fault can be told to its launch.  The switch is read once per process, so a child
process makes the calls, and counts launches and synchronisations in the runtime's trace."""
import os
import subprocess
import sys
from pathlib import Path

import pytest

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parents[1]

CHILD = """
import sys
sys.path.insert(0, %r)
import torch
from torch.profiler import ProfilerActivity, profile
from paper_2608_28511_amd import layer
n = lambda *s: torch.randn(s, device="cuda:0")
bf = lambda *s: n(*s).to(torch.bfloat16)
D, E, F = 64, 8, 48
x, W1, W2 = bf(64, D), bf(E, D, F), bf(E, F, D)
w1, s1 = layer.quant_weights_i8(W1)
w2, s2 = layer.quant_weights_i8(W2)
off = torch.arange(E + 1, dtype=torch.int32, device="cuda:0") * 8
few = [layer.LayerFew(64, n(D, E), W1, W2, 8), layer.LayerFew(64, n(D, E), w1, w2, 8, s1=s1, s2=s2)]
calls = [lambda: few[0](x), lambda: few[1](x), lambda: layer.grouped_ffn_i8(x, off, w1, s1, w2, s2),
         lambda: layer.latent_proj_i8(x, w1[0], s1[0]), lambda: layer.quant_rows_i8(x),
         lambda: layer.quant_weights_i8(W1), lambda: layer.grouped_ffn(x, off, W1, W2)]
for call in calls:
    call()
torch.cuda.synchronize()
for call in calls:
    with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as p:
        call()
    names = [e.name for e in p.events()]
    print("COUNT", sum("LaunchKernel" in v for v in names), sum(v == "hipStreamSynchronize" for v in names))
"""


def counts(switch):
    env = {k: v for k, v in os.environ.items() if k != "MOE_DEBUG_SYNC"}
    if switch:
        env["MOE_DEBUG_SYNC"] = "1"
    r = subprocess.run([sys.executable, "-c", CHILD % str(ROOT)], env=env, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0, r.stderr[-2000:]
    return [tuple(map(int, v.split()[1:])) for v in r.stdout.splitlines() if v.startswith("COUNT")]


def test_every_launch_is_followed_by_a_synchronisation():
    off = counts(False)
    on = counts(True)
    assert len(on) == len(off) == 7
    for (launches, plain), (same, syncs) in zip(off, on):
        assert launches == same and launches >= 1
        assert syncs - plain == launches
