"""A node sweep's work: one training step of the smallest language model there is -- a table of words that is
looked up, projected back onto the vocabulary, and updated -- on every GPU of a node, timed part by part,
checked bit by bit, and scored.

The three parts load three parts of a GPU: the lookup and its gradient scattered rows, the loss and its
gradients the matrix cores, the update the memory's streams.  Every operator gives the same bits for the
same inputs, so two passes from the same start, on one GPU or on eight, must end with the same bits: a
checksum that differs is a GPU that computes wrong numbers.  The parts' rates are what
``Detector.sweep_score`` compares among the eight GPUs.

    python examples/sweep_step.py                                  # one GPU, eight readings of it
    python -m torch.distributed.run --nnodes=1 --nproc-per-node 8 --master-addr 127.0.0.1 \\
        examples/sweep_step.py                                     # the eight GPUs of a node
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_17879_amd import Config, Detector  # noqa: E402

PARTS = ("lookup", "loss", "update")


class SweepStep:
    """The model, its optimizer's states and a batch, made from a seed alone."""

    def __init__(self, det: Detector, rows: int, vocab: int, width: int, bits: int = 32, seed: int = 0):
        self.det, self.rows, self.vocab, self.width, self.bits = det, rows, vocab, width, bits
        dev = det.device
        g = torch.Generator(device=dev)
        g.manual_seed(seed)
        self.start = torch.randn((vocab, width), generator=g, device=dev) * width ** -0.5
        self.tokens = torch.randint(0, vocab, (rows,), generator=g, device=dev)
        self.targets = torch.randint(0, vocab, (rows,), generator=g, device=dev)
        self.targets[::16] = -1                                        # the last words of sequences: no target
        self.master = self.start.clone()
        self.weight = self.master.to(torch.bfloat16)
        self.hidden = torch.empty((rows, width), dtype=torch.bfloat16, device=dev)
        self.grad = {"hidden": torch.empty_like(self.hidden), "weight": torch.empty_like(self.weight)}
        self.out = det.alloc_vocab_loss(rows)
        self.one = torch.ones(1, device=dev)
        self.loss_work = det.alloc_vocab_loss_work(rows, vocab, width, grad=True)
        self.lookup_work = det.alloc_embed_grad_work(rows, vocab, width)
        self.state = det.alloc_adamw_state([self.master], bits)
        self.table = det.adamw_table([self.master], [self.grad["weight"]], self.state, copies=[self.weight],
                                     weight_decay=0.01)
        self.scale = width ** 0.25                                     # logits of a few units, a word's own the largest

    def reset(self):
        """The start once more."""
        self.master.copy_(self.start)
        self.weight.copy_(self.start)
        for tensors in self.state.values():
            for t in tensors:
                t.zero_()

    def lookup(self):
        self.det.embed(self.weight, self.tokens, self.hidden, scale=self.scale)

    def loss(self):
        d = self.det
        d.vocab_loss(self.hidden, self.weight, self.targets, self.out, self.loss_work)
        d.vocab_loss_grad(self.hidden, self.weight, self.targets, self.out, self.grad, self.loss_work,
                          grad_mean=self.one)

    def lookup_grad(self):
        """The table is the projection too: added to the gradient that the loss has left."""
        self.det.embed_grad(self.grad["hidden"], self.tokens, self.grad["weight"], self.lookup_work,
                            scale=self.scale, accumulate=True)

    def update(self, step: int, lr: float):
        self.det.adamw(self.table, lr=lr, step=step)

    def step(self, step: int, lr: float = 1e-3, mark=lambda part: None):
        """One training step; mark(part) is called behind each part."""
        self.lookup()
        mark("lookup")
        self.loss()
        mark("loss")
        self.lookup_grad()
        mark("lookup")
        self.update(step, lr)
        mark("update")

    def checksum(self) -> int:
        """Of everything that a step leaves behind, bit by bit, in 64 bits."""
        total = 0
        for t in (self.master, self.weight, self.hidden, self.grad["hidden"], self.grad["weight"],
                  *self.out.values(), *(x for v in self.state.values() for x in v)):
            b = t.contiguous().view(torch.uint8).view(-1)
            b = torch.cat([b, b.new_zeros(-b.numel() % 4)])
            words = b.view(torch.int32).long() & 0xFFFFFFFF
            # (odd factors: no word that changes alone leaves the sum as it was)
            place = torch.arange(words.numel(), device=words.device) * -0x61C8864680B583EB | 1
            total = (total * 1000003 + int((words * place).sum())) & 0xFFFFFFFFFFFFFFFF
        return total

    def work(self) -> dict:
        """What a step's parts move (bytes) or compute (operations)."""
        counted = int((self.targets >= 0).sum())
        distinct = int(torch.unique(self.tokens).numel())
        row = self.width * 2
        state = 16 if self.bits == 32 else 4
        # there: rows of the table read, looked up ones written; back: their gradients read, the table's read and written
        return {"lookup": 2 * self.rows * 8 + (2 * self.rows + 3 * distinct) * row,
                # the logits of every row; again, and both gradients, of the rows with a target
                "loss": (2.0 * self.rows + 6.0 * counted) * self.vocab * self.width,
                "update": self.vocab * self.width * (4 + 2 + 4 + 2 + state)}


def measure(step: SweepStep, steps: int):
    """Rates of the parts (work per second) over `steps` steps from the start, the losses, and the checksum."""
    step.reset()
    spans = {p: [] for p in PARTS}
    losses = []
    for i in range(1, steps + 1):
        last = [torch.cuda.Event(enable_timing=True)]
        last[0].record()

        def mark(part):
            e = torch.cuda.Event(enable_timing=True)
            e.record()
            spans[part].append((last[0], e))
            last[0] = e

        step.step(i, mark=mark)
        losses.append(step.out["mean"][0].clone())
    torch.cuda.synchronize()
    work = step.work()
    # (the lookup is marked twice a step: there and back)
    seconds = {p: sum(a.elapsed_time(b) for a, b in s) / 1e3 / steps for p, s in spans.items()}
    return {p: work[p] / seconds[p] for p in PARTS}, [float(v) for v in losses], step.checksum()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=65536)
    ap.add_argument("--width", type=int, default=2048)
    ap.add_argument("--bits", type=int, default=32, choices=(8, 32), help="of the optimizer's states")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--tolerance", type=float, default=0.05, help="shortfall against the node's median that is a finding")
    a = ap.parse_args(argv)
    world, rank = int(os.environ.get("WORLD_SIZE", 1)), int(os.environ.get("LOCAL_RANK", 0))
    assert world in (1, 8), "one GPU, or the eight of a node"
    torch.cuda.set_device(rank)
    det = Detector(Config(n_ranks=8, n_metrics=1, window=1, persist_k=1), f"cuda:{rank}")
    step = SweepStep(det, a.rows, a.vocab, a.width, a.bits)
    measure(step, 2)                                                   # warm
    readings = [measure(step, a.steps) for _ in range(8 if world == 1 else 1)]
    if world > 1:
        import torch.distributed as dist
        dist.init_process_group("nccl")
        every = [None] * world
        dist.all_gather_object(every, readings[0])
        readings = every
        dist.destroy_process_group()
    if rank != 0:
        return 0
    rates = torch.tensor([[r[p] for r, _, _ in readings] for p in PARTS], dtype=torch.float32, device=det.device)
    links = torch.ones((len(PARTS), 8, 8), device=det.device)          # (links are another measurement's)
    score = det.sweep_score(rates, links, tol_compute=a.tolerance)
    who = "GPU" if world > 1 else "reading"
    bad = False
    for i, p in enumerate(PARTS):
        unit = "TFLOP/s" if p == "loss" else "GB/s"
        values = "  ".join(f"{v / (1e12 if p == 'loss' else 1e9):8.1f}" for v in rates[i].tolist())
        slow = [g for g in range(8) if int(score["gpu_mask"][i]) >> g & 1]
        bad |= bool(slow)
        print(f"{p:7s} {values} {unit}" + (f"   short: {who} {slow}" if slow else ""))
    sums = [c for _, _, c in readings]
    usual = max(set(sums), key=sums.count)
    wrong = [g for g, c in enumerate(sums) if c != usual]
    losses = readings[0][1]
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps; "
          + (f"WRONG NUMBERS: {who} {wrong}" if wrong else f"all eight {who}s end with the same bits"))
    return 1 if wrong or bad else 0


if __name__ == "__main__":
    sys.exit(main())
