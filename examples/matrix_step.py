"""Training two matrices over sparse exchange, with 8-bit products and orthogonalised steps: every operator of the
library in the order in which a training program calls them.

A network of two square layers with a ReLU between them learns the answers of another one. Each of n workers has its
own inputs; per step

1. the weights are quantised once, by rows for the forward pass and by columns for the backward one (``quantize_i8``);
2. each worker runs both layers (``linear_i8``) and their gradients (``linear_i8_backward``), which leave the weights'
   gradients in binary32;
3. rTop-k with error feedback turns them into messages of k entries (``encode_batch``, one call for all workers and
   both matrices);
4. the master averages the messages, adds them to the momentum, orthogonalises it and moves the weights
   (``aggregate_update_orthogonal``, one call for both matrices).

    python examples/matrix_step.py --width 512 --tokens 1024 --workers 4 --steps 60

All workers share one device here; in a program of one process for each device step 3's messages are what is gathered.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2005_10761_amd as rt  # noqa: E402


class Layer:
    """One matrix, its bias (not trained here) and what its products need."""

    def __init__(self, width, gen, dev):
        self.weights = torch.randn(width, width, device=dev, generator=gen) / width ** 0.5
        self.bias = torch.zeros(width, device=dev)
        self.velocity = torch.zeros(width, width, device=dev)
        # rows of 8-bit numbers start at multiples of 16 bytes
        store = -(-width // 16) * 16
        self.by_rows, self.by_cols = (torch.empty(width, store, dtype=torch.int8, device=dev)[:, :width] for _ in range(2))
        self.row_scale, self.col_scale = torch.empty(width, device=dev), torch.empty(width, device=dev)

    def quantize(self):
        rt.quantize_i8(self.weights, self.by_rows, self.row_scale, along="rows")
        rt.quantize_i8(self.weights, self.by_cols, self.col_scale, along="columns")

    def forward(self, x):
        y = torch.empty_like(x)
        rt.linear_i8(x, self.by_rows, self.row_scale, y, bias=self.bias)
        return y

    def backward(self, dy, x, dw, with_dx):
        dx = torch.empty_like(x) if with_dx else None
        rt.linear_i8_backward(dy, x, self.by_cols if with_dx else None, self.col_scale if with_dx else None, dx, dw)
        return dx


def train(width=512, tokens=1024, workers=4, steps=60, compression=50, eta=0.02, mu=0.9, seed=0, report=None):
    """The mean squared error of all workers at each step."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    layers = [Layer(width, gen, dev) for _ in range(2)]
    answers = [torch.randn(width, width, device=dev, generator=gen) / width ** 0.5 for _ in range(2)]
    d = width * width
    k = max(1, d // compression)
    r = min(d, 5 * k)
    vectors = workers * len(layers)                      # all that is sent in a step: worker 0's matrices, worker 1's, ..
    dw = [[torch.empty(width, width, device=dev) for _ in layers] for _ in range(workers)]
    residual = [torch.zeros(d, device=dev) for _ in range(vectors)]
    # a matrix's messages lie back to back, worker after worker
    idx = [torch.empty(workers * k, dtype=torch.int32, device=dev) for _ in layers]
    val = [torch.empty(workers * k, device=dev) for _ in layers]
    slots = [(w, m) for w in range(workers) for m in range(len(layers))]
    encode_ws = torch.empty(vectors * rt.encode_workspace_bytes(d, r, k), dtype=torch.uint8, device=dev)
    step_ws = torch.empty(rt.aggregate_update_orthogonal_workspace_bytes(len(layers), width, width), dtype=torch.uint8, device=dev)
    losses = []
    for step in range(steps):
        for layer in layers:
            layer.quantize()
        loss = torch.zeros((), device=dev)
        for w in range(workers):
            x = torch.randn(tokens, width, device=dev, generator=gen).to(torch.bfloat16)
            target = torch.relu(x.float() @ answers[0].T) @ answers[1].T
            h = layers[0].forward(x)
            a = torch.relu(h)
            y = layers[1].forward(a)
            error = y.float() - target
            loss += error.square().mean() / workers
            dy = (error * (2.0 / tokens)).to(torch.bfloat16)
            da = layers[1].backward(dy, a, dw[w][1], with_dx=True)
            layers[0].backward(da * (h > 0), x, dw[w][0], with_dx=False)
        rt.encode_batch([dw[w][m] for w, m in slots], residual, r, k, [1000 * seed + i for i in range(vectors)], step,
                        [idx[m][w * k:(w + 1) * k] for w, m in slots], [val[m][w * k:(w + 1) * k] for w, m in slots], encode_ws)
        rt.aggregate_update_orthogonal(idx, val, workers, k, eta, 1.0, mu, [layer.weights for layer in layers],
                                       [layer.velocity for layer in layers], workspace=step_ws)
        losses.append(float(loss))
        if report and (step % 10 == 0 or step == steps - 1):
            report(step, losses[-1])
    return losses


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--width", type=int, default=512, help="inputs, hidden units and outputs")
    p.add_argument("--tokens", type=int, default=1024, help="rows of each worker's inputs in a step")
    p.add_argument("--workers", type=int, default=4)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--compression", type=int, default=50, help="elements of a gradient for each one that is sent")
    a = p.parse_args()
    train(a.width, a.tokens, a.workers, a.steps, a.compression, report=lambda step, loss: print(f"step {step:4d}  loss {loss:.4f}", flush=True))


if __name__ == "__main__":
    main()
