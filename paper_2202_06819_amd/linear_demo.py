"""The linear layer's operators together, as a program uses them.

    python -m paper_2202_06819_amd.linear_demo

Trains a two-layer block on synthetic rows: every layer input is kept for the
backward pass as 8-bit rows (``linear.linear_layer``).  Then serves the trained
block to several requests at once, one token each: its weights as 4-bit rows
shared by all, each request with its own low-rank adapters, the whole step
captured in one graph.  Prints the loss, the bytes kept and the serving error
against 64 bits.
"""
from __future__ import annotations

import torch

from . import linear


class Block:
    """x -> gelu(x W1^T) W2^T with float32 weights, trained through 8-bit rows."""

    def __init__(self, width: int, hidden: int, generator: torch.Generator):
        self.w1, self.w2 = (torch.randn(k, c, generator=generator, device="cuda") * c ** -0.5
                            for k, c in ((hidden, width), (width, hidden)))
        self.w1.requires_grad_()
        self.w2.requires_grad_()

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        return linear.linear_layer(torch.nn.functional.gelu(linear.linear_layer(x, self.w1)), self.w2)


def train(block: Block, width: int, rows: int, steps: int, lr: float, generator: torch.Generator) -> list[float]:
    """Mean squared errors of ``steps`` steps of plain descent towards a fixed random map."""
    target = torch.randn(width, width, generator=generator, device="cuda") * width ** -0.5
    losses = []
    for _ in range(steps):
        x = torch.randn(rows, width, generator=generator, device="cuda").bfloat16()
        loss = (block(x).float() - x.float() @ target).square().mean()
        loss.backward()
        with torch.no_grad():
            for w in (block.w1, block.w2):
                w -= lr * w.grad
                w.grad = None
        losses.append(loss.item())
    return losses


def kept_bytes(block: Block, x: torch.Tensor) -> tuple[int, int]:
    """Bytes the block's linear layers keep for the backward pass of x, and what
    their inputs would take in 16 bits."""
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        block(x)
    inputs = [t for t in kept if t.dtype == torch.int8 and t.shape[0] == x.shape[0]]
    return sum(t.numel() for t in inputs) + 4 * x.shape[0] * len(inputs), 2 * sum(t.numel() for t in inputs)


def rows4(w: torch.Tensor) -> linear.Rows:
    """4-bit rows of weights, the scale fitted to each row's largest value."""
    w = w.detach()
    scale = w.abs().amax(1) / 7.5
    codes = torch.round(w / scale.clamp(min=1e-30)[:, None]).clamp(-8, 7)
    return linear.pack_rows4(codes.to(torch.int8), scale)


class Server:
    """One decoding step of the block for a fixed number of requests, captured."""

    def __init__(self, block: Block, requests: int, adapters: int, rank: int, generator: torch.Generator):
        width, hidden = block.w1.shape[1], block.w1.shape[0]
        self.w1, self.w2 = rows4(block.w1), rows4(block.w2)

        def stack(k, c):
            return linear.Adapters((torch.randn(adapters, rank, c, generator=generator, device="cuda") * c ** -0.5).bfloat16(),
                                   (torch.randn(adapters, k, rank, generator=generator, device="cuda") * 0.1).bfloat16(),
                                   torch.ones(adapters, device="cuda"))
        self.a1, self.a2 = stack(hidden, width), stack(width, hidden)
        self.x = torch.zeros(requests, width, dtype=torch.bfloat16, device="cuda")
        self.row_adapter = torch.full((requests,), -1, dtype=torch.int32, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self._forward()   # the first launches load the kernels
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.y = self._forward()

    def _forward(self) -> torch.Tensor:
        h = linear.linear(linear.quantize_rows(self.x), self.w1, adapters=self.a1, row_adapter=self.row_adapter)
        h = torch.nn.functional.gelu(h)
        return linear.linear(linear.quantize_rows(h), self.w2, adapters=self.a2, row_adapter=self.row_adapter)

    def step(self, x: torch.Tensor, row_adapter: torch.Tensor) -> torch.Tensor:
        self.x.copy_(x)
        self.row_adapter.copy_(row_adapter)
        self.graph.replay()
        return self.y

    def reference(self, x: torch.Tensor, row_adapter: torch.Tensor) -> torch.Tensor:
        """The same with the same weights and adapters in 64 bits, nothing else rounded."""
        def product(x, w, ad):
            nibbles = (w.codes[..., None] >> (4 * torch.arange(8, device="cuda", dtype=torch.int32))) & 15
            values = ((nibbles + 8) & 15) - 8
            values = values.reshape(w.codes.shape[0], -1)[:, :w.channels].double() * w.scale.double()[:, None]
            y = x @ values.t().contiguous()
            for i in range(ad.a.shape[0]):
                mine = (row_adapter == i).nonzero()[:, 0]
                y[mine] += (x[mine] @ ad.a[i].double().t().contiguous()) @ ad.b[i].double().t().contiguous()
            return y
        h = torch.nn.functional.gelu(product(x.double(), self.w1, self.a1))
        return product(h, self.w2, self.a2)


def main(width: int = 256, hidden: int = 1024, rows: int = 2048, steps: int = 40, requests: int = 12, adapters: int = 5,
         rank: int = 16, seed: int = 0) -> dict:
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = Block(width, hidden, g)
    losses = train(block, width, rows, steps, 4.0, g)
    kept, in_16 = kept_bytes(block, torch.randn(rows, width, generator=g, device="cuda").bfloat16())
    server = Server(block, requests, adapters, rank, g)
    worst = 0.0
    for _ in range(3):
        x = torch.randn(requests, width, generator=g, device="cuda").bfloat16()
        ids = torch.randint(-1, adapters, (requests,), generator=g, device="cuda", dtype=torch.int32)
        want = server.reference(x, ids)
        worst = max(worst, float((server.step(x, ids).double() - want).norm() / want.norm()))
    return {"first_loss": losses[0], "last_loss": losses[-1], "kept_bytes": kept, "bytes_in_16_bits": in_16,
            "serving_error": worst}


if __name__ == "__main__":
    for name, value in main().items():
        print(f"{name:18s} {value:.6g}")
