"""What 4-bit weights lose, and how much of it training their scales gives back: a small language model with random weights is the
teacher; the student has its linear layers' weights in 4 bits, and its scales are trained by 4-bit AdamW on the distillation loss
against the teacher's top logits.  Afterwards the student writes a few tokens, one at a time, and is compared with
itself run over the whole text at once.  The student may instead keep its weights, and train them by products with 8-bit operands; gradients may be
clipped, and the tokens drawn instead of the likeliest taken.

    python -m paper_2309_01507_amd.w4_recovery [steps] [--student w4|f8] [--max-norm M] [--temperature T] [--top-p P]
"""
from __future__ import annotations

import argparse
import sys

import torch

from . import binding as B
from .f8 import F8Linear
from .optim import AdamW4bit
from .sampling import sample
from .w4 import W4Linear, distill_loss

VOCAB, WIDTH, INNER, LAYERS, TOKENS, SLOTS, TAU = 5003, 384, 1024, 4, 512, 32, 2.0


class Block(torch.nn.Module):
    """A residual feed-forward block with a running mean of the tokens before, in place of attention"""

    def __init__(self, up, down):
        super().__init__()
        self.up, self.down = up, down

    def forward(self, x, count):
        mean = x.cumsum(0) / count
        h = torch.nn.functional.layer_norm(x + mean, (WIDTH,))
        return x + self.down(torch.nn.functional.gelu(self.up(h)))


class Model(torch.nn.Module):
    def __init__(self, embed, blocks, head):
        super().__init__()
        self.register_buffer("embed", embed)
        self.blocks, self.head = torch.nn.ModuleList(blocks), head

    def forward(self, tokens):
        count = torch.arange(1, tokens.shape[0] + 1, device=tokens.device)[:, None]
        x = self.embed[tokens]
        for b in self.blocks:
            x = b(x, count)
        return self.head(torch.nn.functional.layer_norm(x, (WIDTH,)))

    def write(self, tokens, more: int, temperature: float = 0.0, top_p: float = 1.0, generator=None):
        """`more` tokens behind `tokens`, the likeliest each time or, with a temperature, drawn, by steps of one token; returns them and their logits"""
        sums = [torch.zeros(1, WIDTH, device=tokens.device) for _ in self.blocks]
        out, logits = [], []
        todo = tokens.tolist()
        for at in range(len(todo) + more - 1):
            x = self.embed[todo[at]][None, :]
            for i, b in enumerate(self.blocks):
                sums[i] = sums[i] + x
                h = torch.nn.functional.layer_norm(x + sums[i] / (at + 1), (WIDTH,))
                x = x + b.down(torch.nn.functional.gelu(b.up(h)))
            z = self.head(torch.nn.functional.layer_norm(x, (WIDTH,)))
            if at + 1 >= len(todo):
                todo.append(int(sample(z, temperature, top_p=top_p, generator=generator)[0]) if temperature > 0 else int(z.argmax()))
                out.append(todo[-1])
                logits.append(z)
        return out, torch.cat(logits)


def teacher_model(seed: int, device) -> Model:
    g = torch.Generator(device=device)
    g.manual_seed(seed)

    def linear(n_in, n_out, size):
        layer = torch.nn.Linear(n_in, n_out, bias=False, device=device)
        rows = torch.exp(0.5 * torch.randn(n_out, 1, generator=g, device=device))
        layer.weight.data = size * rows * torch.randn(n_out, n_in, generator=g, device=device) / n_in ** 0.5
        return layer

    embed = torch.randn(VOCAB, WIDTH, generator=g, device=device)
    blocks = [Block(linear(WIDTH, INNER, 1.5), linear(INNER, WIDTH, 1.5)) for _ in range(LAYERS)]
    return Model(embed, blocks, linear(WIDTH, VOCAB, 1.5)).requires_grad_(False)


def student_model(teacher: Model, group: int, kind: str = "w4") -> Model:
    quantized = lambda layer: W4Linear.from_weight(layer.weight, group) if kind == "w4" else F8Linear.from_weight(layer.weight)
    return Model(teacher.embed, [Block(quantized(b.up), quantized(b.down)) for b in teacher.blocks], quantized(teacher.head))


def mean_loss(student, teacher, batches):
    total = 0.0
    with torch.no_grad():
        for tokens in batches:
            top, index = torch.topk(teacher(tokens), SLOTS, dim=1)
            total += float(distill_loss(student(tokens), top, index, TAU).mean())
    return total / len(batches)


def recover(steps: int, seed: int = 0, group: int = 64, lr: float = 2e-4, device="cuda:0", student_kind: str = "w4", max_norm=None, temperature: float = 0.0,
            top_p: float = 1.0):
    """Returns the loss on held-out text before and after, and how far token-by-token logits are from those of the whole text.
    student_kind "f8": the weights themselves are trained, by products with 8-bit operands; max_norm: gradients are clipped to it; temperature, top_p: how
    the text is written."""
    g = torch.Generator(device=device)
    g.manual_seed(seed + 1)
    text = lambda: torch.randint(0, VOCAB, (TOKENS,), generator=g, device=device)
    teacher = teacher_model(seed, device)
    student = student_model(teacher, group, student_kind)
    held_out = [text() for _ in range(4)]
    before = mean_loss(student, teacher, held_out)
    scales = [p for p in student.parameters() if p.requires_grad]
    opt = AdamW4bit(scales, lr=lr, weight_decay=0.0, max_norm=max_norm)
    grad = torch.full((TOKENS,), 1.0 / TOKENS, device=device)
    for _ in range(steps):
        tokens = text()
        top, index = torch.topk(teacher(tokens), SLOTS, dim=1)
        logits = student(tokens)
        _, dz = B.lpmm_distill_loss_grad(logits.detach(), top, index, TAU, grad)      # the mean's gradient is known
        opt.zero_grad()
        logits.backward(dz)
        opt.step()
    after = mean_loss(student, teacher, held_out)
    prompt = held_out[0][:16]
    with torch.no_grad():
        words, logits = student.write(prompt, 8, temperature, top_p, g)
        whole = student(torch.cat([prompt, torch.tensor(words, device=device)]))[len(prompt) - 1:-1]
    return before, after, float((logits - whole).abs().max() / whole.abs().max())


def main(argv):
    arg = argparse.ArgumentParser(prog="w4_recovery")
    arg.add_argument("steps", nargs="?", type=int, default=200)
    arg.add_argument("--student", choices=("w4", "f8"), default="w4")
    arg.add_argument("--max-norm", type=float)
    arg.add_argument("--temperature", type=float, default=0.0)
    arg.add_argument("--top-p", type=float, default=1.0)
    a = arg.parse_args(argv[1:])
    torch.cuda.set_device(0)
    before, after, off = recover(a.steps, student_kind=a.student, max_norm=a.max_norm, temperature=a.temperature, top_p=a.top_p)
    what = "4-bit weights {:.5f}, after {} steps on their scales" if a.student == "w4" else "8-bit products {:.5f}, after {} steps"
    print(f"loss against the teacher's top {SLOTS} logits on held-out text: {what.format(before, a.steps)} "
          f"{after:.5f}; token by token within {off:.1e} of the whole text at once")


if __name__ == "__main__":
    main(sys.argv)
