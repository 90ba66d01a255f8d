"""A small GraphSAGE trainer on the data path (Sec. 4 par. (8); Eq. 1): node classification on a synthetic graph, every
step from a batch's gathered feature block and its computation blocks to new weights.

    python -m paper_2509_05207_amd.train --workload tiny --epochs 4 [--rows8]

The schedule, the cache, the blocks and the feature rows come from the library, and so do the layers' norms with their gradients
(rg_layer_norm, on the gathered rows as they are, padding and all) and the weights' update (rg_muon_step, all matrices in
one call).  Means over neighbours, products and the loss are torch's.

--rows8: features are held in 8 bits in the store, and come through the cache and the gather so (rg_quantize_rows, rg_dequantize_rows), and the layers' products
are those of held rows and held weights (rg_rows8_product), whose backward pass has nothing but the held rows of the forward pass (rg_rows8_product_backward)."""
import argparse
import sys
import time

import torch
from torch.autograd.function import once_differentiable

from . import synth


def layer_norm(rg, eps=1e-5):
    """rg_layer_norm as a function that torch can differentiate, once."""
    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias):
            y, mean, rstd = rg.rg_layer_norm(x, weight, bias, eps=eps)
            ctx.save_for_backward(x, weight, mean, rstd)
            return y

        @staticmethod
        @once_differentiable                              # a second derivative raises: torch does not see into the library's gradients
        def backward(ctx, dy):
            x, weight, mean, rstd = ctx.saved_tensors
            dx, dweight, dbias = ctx.needs_input_grad
            return rg.rg_layer_norm_backward(dy.contiguous(), x, weight, mean, rstd, want_dx=dx, want_dweight=dweight, want_dbias=dbias)
    return Norm.apply


def linear8(rg):
    """x w^T of rows and weights held in 8 bits, as a function that torch can differentiate, once: gradients are those of what the held rows stand for, and the rounding to codes
    counts as the identity.  Only the held rows are kept for the backward pass."""
    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight):
            held, held_weight = rg.rg_quantize_rows(x), rg.rg_quantize_rows(weight)
            ctx.save_for_backward(held, held_weight)
            ctx.cols, ctx.weight_dtype = x.shape[1], weight.dtype
            return rg.rg_rows8_product(held, held_weight, ctx.cols, dtype=x.dtype)

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            held, held_weight = ctx.saved_tensors
            dx, dweight = ctx.needs_input_grad
            return rg.rg_rows8_product_backward(dy.contiguous(), held, held_weight, ctx.cols, want_dx=dx, want_dweight=dweight, want_dbias=False, weight_dtype=ctx.weight_dtype)[:2]
    return Linear.apply


def plain_linear(x, weight):
    return x @ weight.t()


class Sage:
    """L layers h_v <- W [h_v, mean of the sampled neighbours' h], each on normed rows; relu between them."""

    def __init__(self, dim, hidden, n_classes, layers, dtype, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        dims = [dim] + [hidden] * (layers - 1) + [n_classes]
        self.weights = [(torch.randn(o, 2 * i, generator=g, device=device) * (2 * i) ** -0.5).to(dtype).requires_grad_() for i, o in zip(dims, dims[1:])]
        self.scales = [torch.ones(i, device=device).requires_grad_() for i in dims[:-1]]
        self.shifts = [torch.zeros(i, device=device).requires_grad_() for i in dims[:-1]]

    def forward(self, norm, rows, blocks, linear=plain_linear):
        """rows: the batch's feature block; blocks: outermost hop first, (destinations, each edge's destination, each edge's source); linear: a layer's product."""
        h = rows
        for k, (n_dst, dst, src) in enumerate(blocks):
            h = norm(h, self.scales[k], self.shifts[k])
            near = torch.zeros((n_dst, h.shape[1]), dtype=torch.float32, device=h.device).index_add(0, dst, h[src].float())
            degree = torch.bincount(dst, minlength=n_dst).clamp(min=1)
            h = linear(torch.cat([h[:n_dst], (near / degree[:, None]).to(h.dtype)], dim=1), self.weights[k])
            if k + 1 < len(blocks):
                h = torch.relu(h)
        return h


class Muon:
    """rg_muon_step for the matrices, plain descent for the norms' vectors."""

    def __init__(self, rg, model, lr=0.1, weight_decay=0.01, momentum=0.95, vector_lr=0.05):
        self.rg, self.model, self.options, self.vector_lr = rg, model, dict(lr=lr, weight_decay=weight_decay, momentum=momentum), vector_lr
        self.momenta = [torch.zeros(w.shape, dtype=torch.float32, device=w.device) for w in model.weights]
        self.workspace = torch.empty(rg.rg_update_workspace([w.detach() for w in model.weights]), dtype=torch.uint8, device=model.weights[0].device)

    @torch.no_grad()
    def step(self):
        weights = self.model.weights
        self.rg.rg_muon_step([w.detach() for w in weights], [w.grad for w in weights], self.momenta, workspace=self.workspace, **self.options)
        for v in self.model.scales + self.model.shifts:
            v -= self.vector_lr * v.grad
        for p in weights + self.model.scales + self.model.shifts:
            p.grad = None


def held_tables(rg, W, at_once=64 << 20):
    """The feature tables held in 8 bits, where they were: local rows on the device, remote ones there or in pinned host memory.  The latter, which may be too many for the device, by parts of `at_once` bytes."""
    tables = []
    for table in (W.local_rows, W.remote_rows):
        rows = table[:, : W.cfg.feat_dim]
        if table.is_cuda:
            tables.append(rg.rg_quantize_rows(rows))
            continue
        held = synth.pinned_empty((len(rows), rg.rg_rows8_bytes(W.cfg.feat_dim)), torch.uint8)
        part = torch.empty((max(1, min(len(held), at_once // held.shape[1])), held.shape[1]), dtype=torch.uint8, device="cuda")
        for first in range(0, len(held), len(part)):
            n = min(len(part), len(held) - first)
            held[first: first + n].copy_(rg.rg_quantize_rows(rows[first: first + n], out=part[:n]))      # (waits until it is there)
        tables.append(held)
    return tables


class Batches:
    """The batches of one epoch: feature rows, computation blocks and seeds.  held: the feature tables held in 8 bits (held_tables), to be gathered as they are and read back."""

    def __init__(self, rg, W, epoch=0, held=None):
        cfg = W.cfg
        self.rg, self.W, self.held = rg, W, held
        self.schedule = rg.rg_build_schedule(W.indptr, W.indices, W.train, cfg.batch_size, cfg.fanout, cfg.s0, cfg.worker, cfg.epoch + epoch)
        if held is None:
            self.features = rg.make_features(W.is_local, W.row_of, W.local_rows, W.remote_rows, W.row_bytes)
        else:
            self.features = rg.make_features(W.is_local, W.row_of, *held, rg.rg_rows8_bytes(cfg.feat_dim))
        self.cache = rg.rg_build_cache([self.schedule], self.features, W.K)
        rg.rg_schedule_build_blocks(self.schedule)
        s = self.schedule
        self.ids = [rg.rg_schedule_frontier(s, hop) for hop in range(s.L + 1)]
        self.samples = [rg.rg_schedule_samples(s, hop)[0] for hop in range(s.L)]
        self.sources = [rg.rg_schedule_block(s, hop) for hop in range(s.L)]

    def __len__(self):
        return self.schedule.n_batches

    def gathered(self, b):
        """The batch's rows as the gather leaves them: a matrix over padded rows, or held rows."""
        if self.held is None:
            dtype, stride = self.W.local_rows.dtype, self.W.stride_bytes
        else:
            dtype, stride = torch.uint8, self.rg.rg_rows8_bytes(self.W.cfg.feat_dim)
        off = self.ids[-1][2]
        n = int(off[b + 1] - off[b])
        block = torch.empty((n, stride // dtype.itemsize), dtype=dtype, device="cuda")
        self.rg.rg_gather_batch(self.schedule, self.cache, self.features, b, block, out_stride=stride, out_capacity_rows=n, want_stats=False)
        return block

    def rows(self, b):
        """The batch's feature block."""
        block = self.gathered(b)
        if self.held is None:
            return block[:, : self.W.cfg.feat_dim]
        return self.rg.rg_dequantize_rows(block, self.W.cfg.feat_dim, dtype=self.W.local_rows.dtype)

    def blocks(self, b):
        out = []
        for hop in reversed(range(self.schedule.L)):
            off = self.ids[hop][2]
            lo, hi = int(off[b]), int(off[b + 1])
            edges = self.samples[hop][lo: hi + 1]
            first, last = int(edges[0]), int(edges[-1])
            dst = torch.repeat_interleave(torch.arange(hi - lo, device="cuda"), edges[1:] - edges[:-1])
            out.append((hi - lo, dst, self.sources[hop][first:last].long()))
        return out

    def seeds(self, b):
        ids, _, off = self.ids[0]
        return ids[int(off[b]): int(off[b + 1])].long()


def labels_of(W, n_classes, seed=1):
    """A class for every node that its features tell: the largest of n_classes random projections."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    way = torch.randn(W.cfg.feat_dim, n_classes, generator=g, device="cuda")
    local = W.is_local.bool()
    out = torch.empty(W.n_nodes, dtype=torch.long, device="cuda")
    for table, mine in ((W.local_rows, local), (W.remote_rows, ~local)):
        out[mine] = (table[:, : W.cfg.feat_dim].float() @ way).argmax(1)[W.row_of[mine].long()]
    return out


def train_epoch(rg, batches, model, optimiser, labels, norm, linear=plain_linear):
    """One pass; the losses of its batches."""
    losses = []
    for b in range(len(batches)):
        out = model.forward(norm, batches.rows(b), batches.blocks(b), linear)
        loss = torch.nn.functional.cross_entropy(out.float(), labels[batches.seeds(b)])
        loss.backward()
        optimiser.step()
        losses.append(loss.detach())
    return torch.stack(losses)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workload", default="tiny", choices=sorted(c for c, v in synth.CONFIGS.items() if not v.local_rows_only))
    ap.add_argument("--epochs", type=int, default=4)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--classes", type=int, default=16)
    ap.add_argument("--rows8", action="store_true", help="features held in 8 bits, layers' products in 8-bit integers")
    args = ap.parse_args()
    if not torch.cuda.is_available():
        sys.exit("train: no GPU visible; the HIP path has no CPU fallback")
    from . import binding as rg
    rg.lib()
    W = synth.make_workload(args.workload, device="cuda", feature_device="cuda", remote_device="cuda")
    model = Sage(W.cfg.feat_dim, args.hidden, args.classes, len(W.cfg.fanout), W.local_rows.dtype)
    optimiser, norm, labels = Muon(rg, model), layer_norm(rg), labels_of(W, args.classes)
    held, linear = (held_tables(rg, W), linear8(rg)) if args.rows8 else (None, plain_linear)
    for epoch in range(args.epochs):
        t0 = time.perf_counter()
        losses = train_epoch(rg, Batches(rg, W, epoch, held), model, optimiser, labels, norm, linear)
        print(f"epoch {epoch}: loss {losses[0]:.3f} -> {losses[-1]:.3f}, {len(losses)} batches, {time.perf_counter() - t0:.2f} s", flush=True)


if __name__ == "__main__":
    main()
