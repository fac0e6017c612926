"""The package stands on its own: what describes the synthetic workloads is the caller's."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import sys
from types import SimpleNamespace
sys.modules["workloads"] = None                       # an import of it fails
from paper_2501_05370_amd import runner
made = []
class Recorder:
    sdden_mlp4_create = staticmethod(lambda p, group, T, rows: made.append(("mlp4", p, group, T, rows)))
    sdden_gated_create = staticmethod(lambda p, T, rows: made.append(("gated", p, T, rows)))
    sdden_mlp_create = staticmethod(lambda p, T, rows: made.append(("mlp", p, T, rows)))
runner.Denoiser = Recorder
net = SimpleNamespace(d=8, H=8, E=2, W1=0, b1=0, W2=0, b2=0, W3=0, b3=0)
blocks = SimpleNamespace(d=8, H=8, E=2, act=0, eps=1e-5, We=0, be=0, norm_weight=0, norm_bias=0, Wg=0, Wu=0, Wd=0)
four = SimpleNamespace(p=net, group=64)
cfg = SimpleNamespace(kind="mlp", params=net, schedule=None, T=5)
for p in (None, four, blocks):
    runner.make_denoiser(cfg, 7, p)
assert made == [("mlp", net, 5, 7), ("mlp4", net, 64, 5, 7), ("gated", blocks, 5, 7)], made
"""


def test_runner_does_without_the_workloads():
    """Parameters are told apart by their fields, so that a program's own classes do."""
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
