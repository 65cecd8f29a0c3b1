"""A scoring head learns to reproduce the neighbour lists of an index.

    python examples/distill_neighbours.py

An index over encoded vectors answers queries (icq_search); a linear head W [items][features] learns to give each query's
neighbours the scores the index gives them, so that afterwards one product ranks the items.  A step is five calls:
features and weights in 8 bits with a scale per block of 128 (icq_block_quantize), logits as their product (icq_block_matmul),
loss against the search's lists and its gradient in the logits' place (icq_distill), the gradient in 8 bits by rows and by
columns, and the product that gives the weights' gradient.  All buffers are made once; a step allocates nothing.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_1912_08756_amd import binding as icq  # noqa: E402


def neighbour_lists(items=8192, queries=512, d=64, K=8, topk=20, seed=0):
    """(queries [Q][d], ids [Q][topk], distances [Q][topk]) from an index over `items` encoded vectors."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codebooks = torch.randn((K, 256, d), device="cuda", generator=g) * (0.6 ** torch.arange(K, device="cuda"))[:, None, None]
    empty = icq.icq_index_create(codebooks, torch.empty((K, 0), dtype=torch.uint8, device="cuda"), 2)
    x = torch.randn((items, d), device="cuda", generator=g)
    codes = torch.empty((K, items), dtype=torch.uint8, device="cuda")
    icq.icq_encode(empty, x, codes, torch.empty(icq.icq_encode_workspace_bytes(empty, items), dtype=torch.uint8, device="cuda"))
    index = icq.icq_index_create(codebooks, codes, 2)
    q = x[torch.randint(0, items, (queries,), device="cuda", generator=g)] + 0.1 * torch.randn((queries, d), device="cuda", generator=g)
    ids, dist = torch.empty((queries, topk), dtype=torch.int32, device="cuda"), torch.empty((queries, topk), device="cuda")
    everything = torch.full((queries,), float("inf"), device="cuda")
    ws = torch.empty(icq.icq_workspace_bytes(index, queries, items, topk), dtype=torch.uint8, device="cuda")
    icq.icq_search(index, q, everything, items, topk, ids, dist, None, ws)
    return q, ids, dist


class Head:
    """Weights [items][features] in 32 bits, their 8-bit form, and what a step on `rows` rows needs."""

    def __init__(self, items, features, rows, pow2=True):
        dev = dict(device="cuda")
        blocks = lambda n: -(-n // icq.ICQ_BLOCK)
        e4, e5 = torch.float8_e4m3fn, torch.float8_e5m2
        self.pow2 = pow2
        self.weights = torch.zeros((items, features), **dev)
        self.w, self.w_scales = icq.icq_block_codes(items, features), torch.empty((blocks(items), blocks(features)), **dev)
        self.x, self.x_scales = icq.icq_block_codes(rows, features, e4), torch.empty((rows, blocks(features)), **dev)
        self.xt, self.xt_scales = icq.icq_block_codes(features, rows, e4), torch.empty((features, blocks(rows)), **dev)
        self.gt, self.gt_scales = icq.icq_block_codes(items, rows, e5), torch.empty((items, blocks(rows)), **dev)
        self.logits = torch.empty((rows, items), dtype=torch.bfloat16, **dev)
        self.loss, self.grad = torch.empty((rows,), **dev), torch.empty((items, features), **dev)
        need = max(icq.icq_block_matmul_workspace_bytes(rows, items, features), icq.icq_block_matmul_workspace_bytes(items, features, rows),
                   icq.icq_distill_workspace_bytes(rows, items))
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, **dev)

    def scores(self, features):
        icq.icq_block_quantize(features, self.x, self.x_scales, self.xt, self.xt_scales, pow2=self.pow2)
        icq.icq_block_quantize(self.weights, self.w, self.w_scales, block_rows=icq.ICQ_BLOCK, pow2=self.pow2)
        return icq.icq_block_matmul(self.x, self.x_scales, self.w, self.w_scales, self.logits, self.workspace, pow2=self.pow2)

    def step(self, features, ids, dist, temperature, rate):
        """One step of gradient descent; the losses of the rows before it."""
        logits = self.scores(features)
        icq.icq_distill(logits, ids, dist, 1.0, -1.0 / temperature, None, self.loss, grad=logits, workspace=self.workspace)
        icq.icq_block_quantize(logits, None, None, self.gt, self.gt_scales, pow2=self.pow2)
        icq.icq_block_matmul(self.gt, self.gt_scales, self.xt, self.xt_scales, self.grad, self.workspace, pow2=self.pow2)
        self.weights.add_(self.grad, alpha=-rate)
        return self.loss


def train(steps=60, items=8192, queries=512, d=64, features=256, topk=20, temperature=4.0, rate=8.0, seed=0):
    """Mean loss of every step, and the share of queries whose nearest item the head ranks first at the end."""
    q, ids, dist = neighbour_lists(items, queries, d, topk=topk, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.relu(q @ torch.randn((d, features), device="cuda", generator=g))
    x = (x / x.norm(dim=1, keepdim=True)).bfloat16()
    head = Head(items, features, queries)
    losses = [head.step(x, ids, dist, temperature, rate).mean() for _ in range(steps)]
    first = head.scores(x).argmax(1) == ids[:, 0]
    return torch.stack(losses).cpu(), float(first.float().mean())


if __name__ == "__main__":
    torch.cuda.init()
    losses, first = train()
    for k in range(0, len(losses), 10):
        print("step %3d  loss %.4f" % (k, losses[k]))
    print("step %3d  loss %.4f; the index's nearest item ranked first for %.1f %% of the queries" % (len(losses) - 1, losses[-1], 100 * first))
