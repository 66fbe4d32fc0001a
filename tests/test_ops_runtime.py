"""The operators and torch are on one HIP runtime, or the import says that they are not."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)


def test_torch_first():
    p = run("import torch, paper_1610_02496_amd as pk; pk.load_library(); print(pk.ops.layer_norm)")
    assert p.returncode == 0 and "function layer_norm" in p.stdout, p.stdout
    p = run("from paper_1610_02496_amd import ops; print(ops.layer_norm)")
    assert p.returncode == 0 and "function layer_norm" in p.stdout, p.stdout


def test_the_library_first():
    """Without torch the library has loaded the system's runtime, of which torch's streams and memory know nothing; where torch itself
    uses the system's there is only one."""
    code = """
import paper_1610_02496_amd as pk
pk.load_library()
import torch
count = len({line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line})
for attempt in range(2):
    try:
        pk.ops
        print("imported", count)
    except ImportError as e:
        print("refused", count, e)
"""
    p = run(code)
    assert p.returncode == 0, p.stdout
    lines = p.stdout.strip().splitlines()
    assert len(lines) == 2 and all(line.startswith("imported 1") or line.startswith("refused 2") and "import torch before" in line for line in lines), p.stdout
