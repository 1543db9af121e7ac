"""A decode step in planned memory: a few attention layers over 8-bit caches, whose
intermediates are planned once, from the trace of one step, and then live at
their offsets of one slab for every step.

The trace has what a step makes and drops: the projected rows, the selected
blocks, the attention's result, the operators' workspaces, the hidden states between
layers.  What outlives the step is not in it: the caches, which grow by a token a step, are
held in blocks (kv.py), and the last hidden state, which the caller may keep or pass to
the next step, has memory of its own.  The operators write into the planned views, so a step
allocates nothing and can be recorded in a graph.

    python -m paper_2203_00448_amd.decode_step [steps]
"""
from __future__ import annotations

import sys

import torch

from . import binding, kv


class DecodeStep:
    """`layers` attention layers with projections, one token of `n_seqs` sequences a step.

    planned=False gives every intermediate memory of its own: the same step, for comparison."""

    def __init__(self, *, layers=4, n_seqs=8, hidden=512, q_heads=8, heads=2, dim=64, block=16, keep=8,
                 longest=1024, kind=kv.E4M3, planned=True, seed=0):
        self.layers, self.n_seqs, self.hidden = layers, n_seqs, hidden
        self.q_heads, self.heads, self.dim, self.keep = q_heads, heads, dim, keep
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape):
            return torch.randn(shape, generator=gen, device="cuda").mul_(shape[0] ** -0.5).bfloat16()

        rows = q_heads + 2 * heads
        self.w_in = [weight(hidden, rows * dim) for _ in range(layers)]
        self.w_out = [weight(q_heads * dim, hidden) for _ in range(layers)]
        width = (longest + block - 1) // block
        self.caches = [kv.new_cache(n_seqs * width, heads, dim, block=block, kind=kind) for _ in range(layers)]
        order = torch.randperm(n_seqs * width, generator=gen, device="cuda").to(torch.int32)
        self.length = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
        self.seqs = kv.Seqs(order.view(n_seqs, width), self.length, longest=longest)
        self.status = kv.new_status()
        self._lay_out(planned)

    def trace(self):
        """[(name, layer, dtype, shape, first op, last op)] of one step: five ops a layer."""
        n, out = self.n_seqs, []
        spaces = [kv.workspace_size(op, self.caches[0], self.seqs, q_heads=self.q_heads, keep=self.keep)
                  for op in (kv.OP_SELECT, kv.OP_ATTEND)]
        for i in range(self.layers):
            project, _write, select, attend, merge = range(5 * i, 5 * i + 5)
            out += [("rows", i, torch.bfloat16, (n, self.q_heads + 2 * self.heads, self.dim), project, attend),
                    ("blocks", i, torch.int32, (n, self.heads, self.keep), select, attend),
                    ("select_space", i, torch.uint8, (max(16, spaces[0]),), select, select),
                    ("result", i, torch.bfloat16, (n, self.q_heads, self.dim), attend, merge),
                    ("attend_space", i, torch.uint8, (max(16, spaces[1]),), attend, attend),
                    ("added", i, torch.bfloat16, (n, self.hidden), merge, merge)]
            if i < self.layers - 1:
                out.append(("merged", i, torch.bfloat16, (n, self.hidden), merge, merge + 5))
        return out

    def _lay_out(self, planned):
        """The step's tensors: views of one slab at the offsets of a plan, or each its own."""
        trace = self.trace()
        sizes = []
        for _, _, dtype, shape, _, _ in trace:
            count = 1
            for x in shape:
                count *= x
            sizes.append((count * dtype.itemsize + 255) // 256 * 256)
        self.unplanned_bytes = sum(sizes)
        if planned:
            size = torch.tensor(sizes, dtype=torch.int64, device="cuda")
            first = torch.tensor([t[4] for t in trace], dtype=torch.int32, device="cuda")
            last = torch.tensor([t[5] for t in trace], dtype=torch.int32, device="cuda")
            offset, peak = binding.plan_trace(size, first, last, 5 * self.layers)
            _, conflicts, _ = binding.validate_plan(size, first, last, offset)
            assert conflicts == 0
            self.bytes = int(peak.item())
            self.slab, views = binding.apply_plan(offset.tolist(), sizes, self.bytes)
        else:
            self.bytes = self.unplanned_bytes
            views = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in sizes]
        self.at = {}
        for (name, layer, dtype, shape, _, _), view in zip(trace, views):
            count = 1
            for x in shape:
                count *= x
            self.at[name, layer] = view[:count * dtype.itemsize].view(dtype).view(shape)
        self.at["merged", self.layers - 1] = torch.empty(self.n_seqs, self.hidden, dtype=torch.bfloat16, device="cuda")

    def run(self, x):
        """One token of every sequence: x [n_seqs, hidden] in, the last layer's hidden state out.  That
        is one tensor for all steps: the next step's x may be it, and its end writes it again."""
        self.length.add_(1)
        for i, cache in enumerate(self.caches):
            at = {name: self.at[name, i] for name in ("rows", "blocks", "select_space", "result", "attend_space",
                                                      "merged", "added")}
            torch.mm(x, self.w_in[i], out=at["rows"].view(self.n_seqs, -1))
            q = at["rows"][:, :self.q_heads]
            k = at["rows"][:, self.q_heads:self.q_heads + self.heads]
            v = at["rows"][:, self.q_heads + self.heads:]
            kv.write(cache, self.seqs, k, v, status=self.status, check=False)
            kv.select(cache, self.seqs, q, keep=self.keep, first=1, recent=2, out=at["blocks"],
                      workspace=at["select_space"], status=self.status, check=False)
            kv.attend(cache, self.seqs, q, blocks=at["blocks"], out=at["result"],
                      workspace=at["attend_space"], status=self.status, check=False)
            torch.mm(at["result"].view(self.n_seqs, -1), self.w_out[i], out=at["added"])
            torch.add(x, at["added"], out=at["merged"])
            x = at["merged"]
        return x

    def check(self):
        """Waits for the steps so far and raises what any of their calls met."""
        status = int(self.status.item())
        if status != binding.MP_OK:
            raise binding.PlanError(status, "decode step")


def main(steps=300):
    planned, apart = DecodeStep(), DecodeStep(planned=False)
    gen = torch.Generator(device="cuda").manual_seed(1)
    same = True
    for _ in range(steps):
        x = torch.randn(planned.n_seqs, planned.hidden, generator=gen, device="cuda").bfloat16()
        same = same and torch.equal(planned.run(x), apart.run(x))
    planned.check()
    apart.check()
    cached = sum(c.nbytes for c in planned.caches)
    print(f"{steps} steps of {planned.layers} layers: intermediates {planned.bytes} bytes planned, "
          f"{planned.unplanned_bytes} apart; caches {cached} bytes; results "
          f"{'the same' if same else 'DIFFER'}")
    return same


if __name__ == "__main__":
    sys.exit(0 if main(*map(int, sys.argv[1:2])) else 1)
