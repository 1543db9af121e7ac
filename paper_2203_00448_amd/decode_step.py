"""A decode step in planned memory: a few attention layers over caches in 8 or 4 bits, whose
intermediates are planned once, from the trace of one step, and then live at
their offsets of one slab for every step.

The trace has what a step makes and drops: the projected rows, the selected
blocks, the attention's result, the operators' workspaces, the hidden states between
layers.  What outlives the step is not in it: the caches, which grow by a token a step, are
held in blocks (kv.py), their tables and lengths (pages.py), and the last hidden state, which the caller may keep or pass to
the next step, has memory of its own.  The operators write into the planned views, so a step
allocates nothing and can be recorded in a graph.

    python -m paper_2203_00448_amd.decode_step [steps]
"""
from __future__ import annotations

import sys

import torch

from . import binding, kv, pages, rotary


class DecodeStep:
    """`layers` attention layers with projections, one token of `n_seqs` sequences a step.

    keep: blocks that a query reads, 0 for all (a cache in 4 bits, kind E2M1, always has all).
    rotation: a rotary.Rotation by which queries and keys are turned, in place, before they are used.
    paged: blocks are taken from a pool as sequences grow, and `retire` gives back those of sequences that
    ended; otherwise every sequence has its blocks from the start.  Where blocks or a table's room do not suffice for a
    token of every sequence, the step is refused for all: lengths, tables and caches stay as they are, its result
    means nothing, and `check` says so.
    planned=False gives every intermediate memory of its own: the same step, for comparison."""

    def __init__(self, *, layers=4, n_seqs=8, hidden=512, q_heads=8, heads=2, dim=64, block=16, keep=8,
                 longest=1024, kind=kv.E4M3, planned=True, seed=0, rotation=None, paged=False):
        self.layers, self.n_seqs, self.hidden = layers, n_seqs, hidden
        self.q_heads, self.heads, self.dim = q_heads, heads, dim
        self.keep = 0 if kind == kv.E2M1 else keep
        self.rotation, self.paged = rotation, paged
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
        self.table = order.view(n_seqs, width)
        if paged:
            self.pool = pages.Pool(order, torch.zeros(1, dtype=torch.int64, device="cuda"))
            self.table = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
            self.pages_space = pages.workspace(n_seqs)
        # what a step is about: a token more of each sequence, at which positions and places
        self.more = torch.ones(n_seqs, dtype=torch.int32, device="cuda")
        self.step = pages.new_step(n_seqs, n_seqs)
        # what the caches' calls see: the lengths, or zeros in a step that the pool refuses, so that nothing is written
        self.seen = torch.zeros_like(self.length) if paged else self.length
        self.seqs = kv.Seqs(self.table, self.seen, longest=longest)
        self.status = kv.new_status()
        self._lay_out(planned)

    def trace(self):
        """[(name, layer, dtype, shape, first op, last op)] of one step: five ops a layer."""
        n, out = self.n_seqs, []
        spaces = [kv.workspace_size(op, self.caches[0], self.seqs, q_heads=self.q_heads, keep=self.keep)
                  for op in (kv.OP_SELECT, kv.OP_ATTEND)]
        listed = self.keep > 0
        for i in range(self.layers):
            project, _write, select, attend, merge = range(5 * i, 5 * i + 5)
            out.append(("rows", i, torch.bfloat16, (n, self.q_heads + 2 * self.heads, self.dim), project, attend))
            if listed:
                out += [("blocks", i, torch.int32, (n, self.heads, self.keep), select, attend),
                        ("select_space", i, torch.uint8, (max(16, spaces[0]),), select, select)]
            out += [("result", i, torch.bfloat16, (n, self.q_heads, self.dim), attend, merge),
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
        if self.paged:
            pages.extend(self.pool, self.table, self.length, self.more, block=self.caches[0].block, step=self.step,
                         workspace=self.pages_space, status=self.status, check=False)
            # the tokens before the second sequence: one, none on a refusal.  (As bounds of the calls, which look
            # for a row's sequence then, a step of 8 sequences took 108 us for 105 in 4 bits, 158 for 138 in 8.)
            torch.mul(self.length, self.step.begin[1:2], out=self.seen)
        else:
            self.length.add_(1)
            if self.rotation is not None:
                torch.sub(self.length, 1, out=self.step.position)
        for i, cache in enumerate(self.caches):
            at = {name: self.at.get((name, i)) for name in ("rows", "blocks", "select_space", "result",
                                                            "attend_space", "merged", "added")}
            torch.mm(x, self.w_in[i], out=at["rows"].view(self.n_seqs, -1))
            q = at["rows"][:, :self.q_heads]
            k = at["rows"][:, self.q_heads:self.q_heads + self.heads]
            v = at["rows"][:, self.q_heads + self.heads:]
            if self.rotation is not None:
                rotary.rotate(self.rotation, self.step.position, q, k, out=q, k_out=k)
            kv.write(cache, self.seqs, k, v, status=self.status, check=False)
            if self.keep:
                kv.select(cache, self.seqs, q, keep=self.keep, first=1, recent=2, out=at["blocks"],
                          workspace=at["select_space"], status=self.status, check=False)
            kv.attend(cache, self.seqs, q, blocks=at["blocks"], out=at["result"],
                      workspace=at["attend_space"], status=self.status, check=False)
            torch.mm(at["result"].view(self.n_seqs, -1), self.w_out[i], out=at["added"])
            torch.add(x, at["added"], out=at["merged"])
            x = at["merged"]
        return x

    def retire(self, done):
        """Sequences with done bool [n_seqs] set start anew; their blocks go back to the pool."""
        if not self.paged:
            raise ValueError("only blocks of a pool go back")
        pages.release(self.pool, self.table, self.length, done, block=self.caches[0].block,
                      workspace=self.pages_space, status=self.status, check=False)

    def check(self):
        """Waits for the steps so far and raises what any of their calls met."""
        status = int(self.status.item())
        if status != binding.MP_OK:
            raise binding.PlanError(status, "decode step")


def compare(steps, what, **options):
    """Steps in planned memory beside the same ones with memory of their own."""
    planned, apart = DecodeStep(**options), DecodeStep(planned=False, **options)
    gen = torch.Generator(device="cuda").manual_seed(1)
    same = True
    for _ in range(steps):
        x = torch.randn(planned.n_seqs, planned.hidden, generator=gen, device="cuda").bfloat16()
        same = same and torch.equal(planned.run(x), apart.run(x))
    planned.check()
    apart.check()
    cached = sum(c.nbytes for c in planned.caches)
    print(f"{what}: {steps} steps of {planned.layers} layers: intermediates {planned.bytes} bytes planned, "
          f"{planned.unplanned_bytes} apart; caches {cached} bytes; results "
          f"{'the same' if same else 'DIFFER'}")
    return same


def main(steps=300):
    same = compare(steps, "8 bits, selected blocks")
    return compare(steps, "4 bits, rotary positions, blocks from a pool", kind=kv.E2M1, paged=True,
                   rotation=rotary.Rotation(64)) and same


if __name__ == "__main__":
    sys.exit(0 if main(*map(int, sys.argv[1:2])) else 1)
