"""A plan that does not fit the host's memory is an error that the caller sees, not the end of the process."""
import subprocess
import sys
from pathlib import Path

CHILD = """
import resource, sys
import numpy as np
import paper_2502_02534_b200 as psa
psa.library()
n = 1 << 23
small = psa.Plan([64], [2], [5, 40], num_q_heads=8, num_kv_heads=8, head_dim=64, num_sms=148)
lens = np.full(n, 4096, np.int32)
plan = psa.Plan([0], [n], np.zeros(n, np.int32), num_q_heads=8, num_kv_heads=8, head_dim=64, num_sms=148) if sys.argv[1] == "kv4" else None
with open("/proc/self/statm") as f:
    now = int(f.read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (now + (64 << 20), resource.getrlimit(resource.RLIMIT_AS)[1]))
try:
    if plan is not None:
        plan.for_kv4()
    else:
        psa.Plan([0], [n], lens, num_q_heads=8, num_kv_heads=8, head_dim=64, num_sms=148)
    print("made")
except psa.PsaError as e:
    print("refused:", e)
print(small.for_kv4().info.num_samples)
"""


def run(kind):
    return subprocess.run([sys.executable, "-c", CHILD, kind], capture_output=True, text=True, timeout=120, cwd=Path(__file__).resolve().parent.parent)


def test_plans():
    for kind in ("bf16", "kv4"):
        r = run(kind)
        assert r.returncode == 0 and "refused" in r.stdout and "memory" in r.stdout and r.stdout.endswith("2\n"), (kind, r.returncode, r.stdout, r.stderr[-500:])
