"""A scoring head learns to reproduce the neighbour lists of an index.

    python examples/distill_neighbours.py [--bits 4]

An index over encoded vectors answers queries (icq_search); a linear head W [items][features] learns to give each query's
neighbours the scores the index gives them, so that afterwards one product ranks the items.  A step is five calls:
features and weights in 8 bits with a scale per block of 128 (icq_block_quantize), logits as their product (icq_block_matmul),
loss against the search's lists and its gradient in the logits' place (icq_distill), the gradient in 8 bits by rows and by
columns, and the product that gives the weights' gradient.  All buffers are made once; a step allocates nothing.

With --bits 4 the head is held in microscaled 4-bit floating point (icq_mx_quantize, icq_mx_matmul), has a bias for each item, and its gradients are
clipped by their global norm before the update (icq_grad_norm_clip).
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


class MxHead:
    """Weights [items][features] and a bias for each item in 32 bits, the weights' 4-bit form, and what a step on `rows` rows needs.  A step changes weights
    and bias, not the 4-bit form: hold() after the last one brings it up to date, and answer() gives scores of that head."""

    def __init__(self, items, features, rows, max_norm=float("inf")):
        dev = dict(device="cuda")
        held = lambda r, c: (icq.icq_mx_codes(r, c), icq.icq_mx_scales(r, c))
        self.max_norm = max_norm
        self.weights, self.bias = torch.zeros((items, features), **dev), torch.zeros((items,), **dev)
        self.w, self.x, self.xt, self.gt = held(items, features), held(rows, features), held(features, rows), held(items, rows)
        self.logits, self.loss = torch.empty((rows, items), dtype=torch.bfloat16, **dev), torch.empty((rows,), **dev)
        self.grad, self.bias_grad, self.norm = torch.empty((items, features), **dev), torch.empty((items,), **dev), torch.empty((1,), **dev)
        self.grads = icq.icq_grad_list_create([self.grad, self.bias_grad])
        need = max(icq.icq_mx_matmul_workspace_bytes(rows, items, features), icq.icq_mx_matmul_workspace_bytes(items, features, rows),
                   icq.icq_distill_workspace_bytes(rows, items), icq.icq_grad_workspace_bytes(self.grads))
        self.workspace = torch.empty(max(need, 256), dtype=torch.uint8, **dev)
        self.hold()

    def hold(self):
        """The weights' 4-bit form, from the weights as they are now."""
        icq.icq_mx_quantize(self.weights, *self.w, block_rows=icq.ICQ_MX_BLOCK, fit=True)

    def scores(self, features):
        icq.icq_mx_quantize(features, *self.x, *self.xt, fit=True)
        self.hold()
        icq.icq_mx_matmul(*self.x, *self.w, self.logits, self.workspace, K=features.shape[1])
        return self.logits.add_(self.bias)

    def answer(self, features):
        """Scores of any number of rows, mostly a few, from the weights as they are held and the bias, the features quantised on the way."""
        rows, items = features.shape[0], self.bias.numel()
        out = torch.empty((rows, items), device="cuda")
        need = icq.icq_mx_matmul_workspace_bytes(rows, items, features.shape[1], features.dtype)
        space = self.workspace if need <= self.workspace.numel() else torch.empty(need, dtype=torch.uint8, device="cuda")
        return icq.icq_mx_matmul(features, None, *self.w, out, space, K=features.shape[1], fit=True).add_(self.bias)

    def step(self, features, ids, dist, temperature, rate):
        """One step of gradient descent; the losses of the rows before it."""
        logits = self.scores(features)
        icq.icq_distill(logits, ids, dist, 1.0, -1.0 / temperature, None, self.loss, grad=logits, workspace=self.workspace)
        icq.icq_mx_quantize(logits, None, None, *self.gt, fit=True)
        icq.icq_mx_matmul(*self.gt, *self.xt, self.grad, self.workspace, K=features.shape[0])
        torch.sum(logits, 0, dtype=torch.float32, out=self.bias_grad)
        icq.icq_grad_norm_clip(self.grads, self.norm, self.max_norm, self.workspace)
        self.weights.add_(self.grad, alpha=-rate)
        self.bias.add_(self.bias_grad, alpha=-rate)
        return self.loss


def train(steps=60, items=8192, queries=512, d=64, features=256, topk=20, temperature=4.0, rate=8.0, seed=0, bits=8):
    """Mean loss of every step, and the share of queries whose nearest item the head ranks first at the end."""
    q, ids, dist = neighbour_lists(items, queries, d, topk=topk, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x = torch.relu(q @ torch.randn((d, features), device="cuda", generator=g))
    x = (x / x.norm(dim=1, keepdim=True)).bfloat16()
    head = Head(items, features, queries) if bits == 8 else MxHead(items, features, queries, max_norm=1.0)
    losses = [head.step(x, ids, dist, temperature, rate).mean() for _ in range(steps)]
    first = head.scores(x).argmax(1) == ids[:, 0]
    return torch.stack(losses).cpu(), float(first.float().mean())


if __name__ == "__main__":
    torch.cuda.init()
    losses, first = train(bits=4 if sys.argv[1:] == ["--bits", "4"] else 8)
    for k in range(0, len(losses), 10):
        print("step %3d  loss %.4f" % (k, losses[k]))
    print("step %3d  loss %.4f; the index's nearest item ranked first for %.1f %% of the queries" % (len(losses) - 1, losses[-1], 100 * first))
