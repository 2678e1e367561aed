"""The status word of losses and products that are given none."""

import subprocess
import sys

import pytest
import torch

from paper_2607_13332_b200 import binding, stage_ops

pytestmark = pytest.mark.gpu


def inputs():
    logits = torch.randn(5, 300, device="cuda")
    ids = torch.arange(15, dtype=torch.int32, device="cuda").view(5, 3)
    return logits, ids, torch.randn(5, 3, device="cuda")


def test_an_id_outside_the_vocabulary_is_on_record():
    logits, ids, top = inputs()
    stage_ops.take_status()
    stage_ops.distill_loss_grad(logits, ids, top)
    assert stage_ops.take_status() == 0
    ids[2, 1] = 300
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        stage_ops.distill_loss(logits, ids, top)
    assert stage_ops.take_status() == binding.SSN_DEV_BAD_ID and stage_ops.take_status() == 0
    stage_ops.distill_loss_grad(logits, ids, top)
    assert stage_ops.take_status() == binding.SSN_DEV_BAD_ID
    own = torch.zeros(1, dtype=torch.int32, device="cuda")      # a word of the caller's: the library's stays as it is
    stage_ops.distill_loss(logits, ids, top, dev_status=own)
    assert int(own) == binding.SSN_DEV_BAD_ID and stage_ops.take_status() == 0


def test_products_leave_it_alone():
    q, s = stage_ops.int8_quantize(torch.randn(300, 512, device="cuda"))
    stage_ops.take_status()
    for n in (1, 40, 300):
        stage_ops.int8_matmul(q[:n], s[:n], q, s)
    assert stage_ops.take_status() == 0


FIRST_IN_A_CAPTURE = """
import torch
from paper_2607_13332_b200 import binding, stage_ops
logits, top = torch.randn(5, 300, device="cuda"), torch.randn(5, 3, device="cuda")
ids = torch.full((5, 3), 400, dtype=torch.int32, device="cuda")
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    loss, grad = stage_ops.distill_loss_grad(logits, ids, top)
for _ in range(2):
    graph.replay()
    assert stage_ops.take_status() == binding.SSN_DEV_BAD_ID
    assert stage_ops.take_status() == 0
print("recorded", int(grad.any()))
"""


def test_a_process_whose_first_call_is_captured():
    got = subprocess.run([sys.executable, "-c", FIRST_IN_A_CAPTURE], capture_output=True, text=True, timeout=300)
    assert got.returncode == 0 and "recorded 0" in got.stdout, got.stderr[-1500:]
