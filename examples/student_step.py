"""A distillation step of a student, its body's activations kept in 8 bits: pre-normed feed-forward blocks (gate and up
projection, gated activation, down projection), a norm, a gate per channel and a residual scale after each block, and
the fused chunked KL loss over the LM head.

    python examples/student_step.py                       # peak memory and time, 8-bit records against plain tensors
    python examples/student_step.py --tokens 65536 --layers 8 --act8 e4m3

Random weights and synthetic hidden states; the arithmetic, the shapes and the memory are a real step's. The bf16 side's
activation is two eager torch operations, which keep the activated gate as well and are slower than gated_act's kernels.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_03796_b200.autograd import act8_linear, block_norm, check_status, fused_chunked_kl, gated_act  # noqa: E402


class Block(torch.nn.Module):
    """W_down (act(W_gate y) * (W_up y)), then the join with the residual stream and the norm for the next block."""

    def __init__(self, H, F, branch_scale, device, generator):
        super().__init__()

        def weight(n, k):
            return torch.nn.Parameter((torch.randn(n, k, generator=generator, device=device) / k ** 0.5).bfloat16())
        self.gate_up, self.down = weight(2 * F, H), weight(H, F)
        ones = torch.ones(H, dtype=torch.bfloat16, device=device)
        self.post, self.pre, self.gate = (torch.nn.Parameter(t) for t in (ones.clone(), ones.clone(), 0.5 * ones))
        self.branch_scale = branch_scale

    def forward(self, y, kept, x, act8):
        """(y, record of y, x) in and out: the normed input, its 8-bit record if there is one, the residual stream."""
        args = dict(eps=1e-5, branch_scale=self.branch_scale)
        if act8 is None:
            gate, up = torch.nn.functional.linear(y, self.gate_up).chunk(2, dim=-1)
            branch = torch.nn.functional.linear(torch.nn.functional.silu(gate) * up, self.down)
            y, x = block_norm(x, branch, self.post, self.pre, self.gate, **args)
            return y, None, x
        h, kept_h = gated_act(act8_linear(y, self.gate_up, record=kept, act8=act8), act="silu", act8=act8, keep_h=True)
        branch = act8_linear(h, self.down, record=kept_h, act8=act8)
        y, x, kept = block_norm(x, branch, self.post, self.pre, self.gate, act8=act8, keep_y=True, **args)
        return y, kept, x


class Student(torch.nn.Module):
    def __init__(self, H, F, V, layers, device="cuda", seed=0):
        super().__init__()
        g = torch.Generator(device=device).manual_seed(seed)
        self.blocks = torch.nn.ModuleList(Block(H, F, (2 * layers) ** -0.5, device, g) for _ in range(layers))
        self.first = torch.nn.Parameter(torch.ones(H, dtype=torch.bfloat16, device=device))
        self.head = torch.nn.Parameter((torch.randn(V, H, generator=g, device=device) / H ** 0.5).bfloat16())

    def forward(self, x, act8):
        """The hidden states [T, H] that the LM head reads."""
        y, _ = block_norm(x, torch.zeros_like(x), pre_weight=self.first, eps=1e-5)
        kept = None
        for block in self.blocks:
            y, kept, x = block(y, kept, x, act8)
        return y


def step(student, x, teacher, act8, chunk=4096):
    """Loss of one step; the gradients are left in the parameters."""
    idx, val = teacher
    loss = fused_chunked_kl(student(x, act8), student.head, idx, val, chunk=chunk)
    loss.backward()
    return loss.detach()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("tokens", 32768), ("hidden", 2048), ("ffn", 5632), ("vocab", 32768), ("layers", 4), ("steps", 5)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--act8", default="int8", choices=["int8", "e4m3"])
    a = ap.parse_args()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.tokens, a.hidden, generator=g, device="cuda").bfloat16()
    idx = torch.randint(0, a.vocab, (a.tokens, 64), generator=g, device="cuda", dtype=torch.int32)
    val = 3 * torch.randn(a.tokens, 64, generator=g, device="cuda")
    grads = {}
    for act8 in (None, a.act8):
        student = Student(a.hidden, a.ffn, a.vocab, a.layers)
        for _ in range(2):
            student.zero_grad(set_to_none=True)
            loss = step(student, x, (idx, val), act8)
        torch.cuda.synchronize()
        student.zero_grad(set_to_none=True)
        held = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        began = time.perf_counter()
        for _ in range(a.steps):
            student.zero_grad(set_to_none=True)
            step(student, x, (idx, val), act8)
        torch.cuda.synchronize()
        ms = (time.perf_counter() - began) / a.steps * 1e3
        check_status()
        peak = torch.cuda.max_memory_allocated() - held
        print(f"activations {act8 or 'bf16'}: loss {loss.item():.6f}, {ms:.1f} ms a step, {peak / 2 ** 30:.2f} GiB of "
              "activations and gradients at most")
        grads[act8] = {n: p.grad.float() for n, p in student.named_parameters()}
        del student
    off = {n: ((grads[a.act8][n] - v).norm() / v.norm()).item() for n, v in grads[None].items()}
    worst = max(off, key=off.get)
    print(f"gradients against those from bf16 activations: {max(off.values()):.4f} relative at most ({worst})")


if __name__ == "__main__":
    main()
