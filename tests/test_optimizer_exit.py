"""A program that ends with an AdamW optimizer's plan alive ends without a word, and plans are freed before that too."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import torch
from paper_2511_12653_amd import AdamW, binding as fq, optim
torch.cuda.current_stream = lambda *_: None
destroyed, destroy = [], fq.fq_adamw_destroy
def counted(handle):
    destroyed.append(handle)
    destroy(handle)
fq.fq_adamw_destroy = counted
create = fq.fq_adamw_create
fq.fq_adamw_create = lambda params, workspace: create(params, workspace, stream=0)
opt = AdamW([{"params": []}])
plan = lambda: optim._Plan((), [], [], [], [], "cpu")      # (of an empty list: no GPU is involved)
opt._plans[0, 0] = plan()
opt._plans[0, 0] = plan()
print("destroyed", len(destroyed))
opt._plans.clear()
print("destroyed", len(destroyed))
opt._plans[0, 0] = plan()
"""


def test_the_end_of_a_program_is_quiet():
    got = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=200)
    assert got.returncode == 0 and got.stdout.split() == ["destroyed", "1", "destroyed", "2"], got.stdout + got.stderr
    assert "Exception ignored" not in got.stderr and "Traceback" not in got.stderr, got.stderr
