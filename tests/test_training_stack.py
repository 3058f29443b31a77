"""A call with many tensors runs on a thread with a small stack: the 32 KB table of their records is neither there nor copied there.
(In a child process that sees no GPU, so that the launches come back with an error at once.)"""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import sys, threading
sys.path.insert(0, sys.argv[1])
from paper_2609_36074_b200 import training
fn = training._load()["clip_grad_norm"]
count, chunks, got = int(sys.argv[2]), int(sys.argv[3]), []
t = (training.Tensor * count)(*[(1 << 20, 2 << 20, chunks * 2048, 0, 0)] * count)
call = lambda: got.append(fn(t, count, 1.0, 1e-6, 1 << 20, 1 << 20, 1 << 30, None))
call()                                      # what is set up on a first call may take what it likes
threading.stack_size(64 << 10)
th = threading.Thread(target=call)
th.start()
th.join()
print(got)
"""


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses: only where nothing can be launched")
@pytest.mark.parametrize("count,chunks", [(1000, 1), (1000, 50), (3000, 1), (65, 0), (64, 1)])
def test_many_tensors_on_a_small_stack(count, chunks):
    child = subprocess.run([sys.executable, "-c", CHILD, ROOT, str(count), str(chunks)], env={**os.environ, "CUDA_VISIBLE_DEVICES": ""},
                           capture_output=True, text=True, timeout=300)
    assert child.returncode == 0 and child.stdout.strip() == "[-2, -2]", (child.returncode, child.stdout, child.stderr[-500:])
