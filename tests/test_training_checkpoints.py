"""What the binding asks of a checkpoint before the library reads its memory: that it is there, on a GPU, as large as its shape needs, also in
a process that has packed none itself and without assertions."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2309_06497_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def kept(rows=4, cols=40, code=B.GRAD_F32, nbytes=None):
    """On the CPU, as from a file"""
    n = B.lib().shampoo_checkpoint_bytes(rows, cols) if nbytes is None else nbytes
    return B.Checkpoint(torch.zeros(n, dtype=torch.uint8), (rows, cols), code)


READERS = r"""
import torch
from paper_2309_06497_amd import binding as B
from tests.test_training_checkpoints import kept
c, x = kept(), torch.zeros((4, 40))
calls = [lambda: B.shampoo_checkpoint_unpack(c), lambda: B.shampoo_checkpoint_activation_grad(c, x, B.ACT_RELU),
         lambda: B.shampoo_checkpoint_weight_grad(c, x), lambda: B.shampoo_checkpoint_unpack(c, dtype=torch.bfloat16),
         lambda: B.shampoo_residual_norm_backward(c, c, None, x, w_post=x[0], w_pre=x[0]),
         lambda: B.shampoo_residual_norm_backward(c, kept(5), None, x, w_post=x[0], w_pre=x[0]),
         lambda: B.shampoo_residual_norm_backward(c, kept(code=B.GRAD_BF16), None, x, w_post=x[0], w_pre=x[0]),
         lambda: B.shampoo_residual_norm_backward(c, x, None, x, w_post=x[0], w_pre=x[0]),
         lambda: B.shampoo_residual_norm_backward(x, c, None, x, w_post=x[0], w_pre=x[0])]
for i in WHICH:
    try:
        calls[i]()
        print("accepted")
    except Exception as e:
        print(type(e).__name__, e)
print(c.dtype)
"""


@pytest.mark.parametrize("flags,which", [([], [k]) for k in range(4)] + [([], []), ([], list(range(9))), (["-O"], list(range(8, -1, -1)))])
def test_a_checkpoint_that_a_process_has_not_packed(flags, which):
    env = dict(os.environ, PYTHONPATH=ROOT)
    p = subprocess.run([sys.executable] + flags + ["-c", READERS.replace("WHICH", str(which))], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0, p.stderr[-2000:]
    lines = p.stdout.split("\n")
    assert lines[len(which)] == "torch.float32"
    for line in lines[:len(which)]:
        assert line.startswith("AssertionError ") and len(line) > 16, lines       # refused by name, with a reason


@pytest.mark.gpu
def test_a_checkpoint_whose_memory_does_not_hold_its_shape():
    x = torch.randn((70, 200), device="cuda")
    c, other = B.shampoo_checkpoint_pack(x), B.shampoo_checkpoint_pack(x)
    w = torch.ones(200, device="cuda")
    held = c.packed
    spaced = torch.zeros((held.numel(), 2), dtype=torch.uint8, device="cuda")[:, 0]
    for memory in (held[:-1], held[:0], held.cpu(), held.view(torch.int8), held[:held.numel() // 8 * 8].view(torch.float64), spaced, None):
        bad = B.Checkpoint(memory, (70, 200), B.GRAD_F32)
        for call in (lambda: B.shampoo_checkpoint_unpack(bad), lambda: B.shampoo_checkpoint_activation_grad(bad, x, B.ACT_SILU),
                     lambda: B.shampoo_checkpoint_weight_grad(bad, x), lambda: B.shampoo_residual_norm_backward(bad, other, x, x, w_post=w, w_pre=w),
                     lambda: B.shampoo_residual_norm_backward(other, bad, x, x, w_post=w, w_pre=w)):
            with pytest.raises(AssertionError):
                call()
    for rows, cols in ((71, 200), (70, 201), (70, 225), (-1, 200), (70, 0), (70, -200), (70, (1 << 32) + 200)):
        if B.lib().shampoo_checkpoint_bytes(rows, min(cols, 1 << 20)) <= held.numel() and 0 < cols < 1 << 31 and rows >= 0:
            continue                                    # inside the same padding
        with pytest.raises(AssertionError):
            B.shampoo_checkpoint_unpack(B.Checkpoint(held, (rows, cols), B.GRAD_F32))
    for activation in (4, -1):
        with pytest.raises(B.ShampooError):
            B.shampoo_checkpoint_unpack(c, activation)
    with pytest.raises(AssertionError):
        B.shampoo_checkpoint_unpack(c, 1 << 32)
    # moved and moved back: the same
    again = B.Checkpoint(held.cpu().cuda(), (70, 200), B.GRAD_F32)
    assert torch.equal(B.shampoo_checkpoint_unpack(again), B.shampoo_checkpoint_unpack(c))
