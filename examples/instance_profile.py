#!/usr/bin/env python3
"""A hardware profile measured on this GPU, and the plan it leads to.

The scheduler's estimator needs, for every class of instances and every model,
the seconds of a prompt (P), the seconds of a decode step (d) and the tokens that
the memory holds (GPU) -- Sec. 6, "Offline profiling".  Here an instance of this
GPU is run instead of described: a stack of decoder layers with random 4-bit
weights (qlm.w4_matmul) over an 8-bit token cache (qlm.kv_append,
qlm.kv_attention) whose sequences give up their least attended tokens when they
pass a budget (qlm.kv_evict).  With --bits 8 the weights are in 8-bit floating point
(qlm.f8_rows, qlm.f8_matmul); with --drafts N a step checks N drafted tokens of every
sequence (qlm.draft_verify), keys and queries turned by their positions
(qlm.kv_append_rotated), and a token's seconds are the step's over the tokens that it
gave.  The measured numbers go through qlm.apply_profile
into the tables of a scheduling problem, and qlm.best_plan picks a plan.

    python examples/instance_profile.py [--layers 32] [--batch 32] ...
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2407_00047_amd import qlm, workload  # noqa: E402

BLOCK = qlm.KV_BLOCK


class Model:
    """Sizes of a decoder layer and the 4-bit (or 8-bit) weights of a stack of them.  Every
    layer has the same codes, as the time of a step does not depend on them, in memory
    of its own: a step reads each layer's weights anew, where one layer's would come from the
    last-level cache (90 MB at the sizes below, of 256)."""

    def __init__(self, hidden, heads, kv_heads, dim, inner, group=128, seed=0, layers=1, bits=4,
                 vocab=0):
        self.hidden, self.heads, self.kv_heads, self.dim = hidden, heads, kv_heads, dim
        self.inner, self.vocab = inner, vocab
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def matrix(n_out, n_in):
            if bits == 8:
                # (normal weights in units of a 110th: the largest of a block near code 448)
                codes = (110.0 * torch.randn((n_out, n_in), generator=gen, device="cuda"))
                scale = torch.full((-(-n_out // qlm.F8_BLOCK), -(-n_in // qlm.F8_BLOCK)),
                                   n_in ** -0.5 / 110, device="cuda")
                return qlm.f8_pack(codes.clamp(-448, 448).to(torch.float8_e4m3fn), scale)
            codes = torch.randint(0, 16, (n_out, n_in), generator=gen, device="cuda",
                                  dtype=torch.uint8)
            groups = -(-n_in // group)
            scale = torch.full((n_out, groups), 0.2 * n_in ** -0.5, device="cuda").half()
            zero = torch.randint(7, 9, (n_out, groups), generator=gen, device="cuda",
                                 dtype=torch.uint8)
            return qlm.w4_pack(codes, scale, zero, group)

        first = (matrix((heads + 2 * kv_heads) * dim, hidden), matrix(hidden, heads * dim),
                 matrix(inner, hidden), matrix(hidden, inner))
        copy = lambda m: (qlm.F8(m.packed.clone(), m.n_out, m.n_in) if bits == 8 else  # noqa: E731
                          qlm.W4(m.packed.clone(), m.n_out, m.n_in, m.group))
        # (qkv, out, up, down) of each layer
        self.layers = [first] + [tuple(copy(m) for m in first) for _ in range(layers - 1)]

        if vocab:                      # words' vectors, and the product that scores the words
            self.words = torch.randn((vocab, hidden), generator=gen, device="cuda").bfloat16()
            self.head = matrix(vocab, hidden)

    def weight_bytes(self, layers):
        return layers * sum(m.packed.numel() for m in self.layers[0])

    def token_bytes(self, layers):
        """Cache bytes of a token: codes of keys and values, its position and weight,
        its part of the block scales."""
        return layers * self.kv_heads * (2 * self.dim + 8 + 8 / BLOCK)


class Instance:
    """Sequences in decode on one model: their cache, a block table and lengths."""

    def __init__(self, model, layers, batch, most, positions=0):
        if layers > len(model.layers):
            raise ValueError("the model has %d layers" % len(model.layers))
        self.model, self.layers, self.batch = model, layers, batch
        self.width = -(-most // BLOCK)
        n = batch * self.width
        self.caches = [qlm.DeviceKvCache.empty(n, model.kv_heads, model.dim)
                       for _ in range(layers)]
        order = torch.randperm(n, device="cuda").int()
        self.table = order.view(batch, self.width).contiguous()
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.next = torch.zeros(batch, dtype=torch.int32, device="cuda")   # next position
        # the same, known to the host (behind drafted steps more: refused drafts count too)
        self.position = 0
        self.rotary = None
        if positions:                  # keys and queries are turned by their positions
            pairs = model.dim // 2
            freq = 10000.0 ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
            angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * freq
            self.rotary = qlm.Rotary(angle.cos().float(), angle.sin().float())
        self.ws = {}

    def _workspace(self, name, need, make):
        """One workspace for each use, grown when a larger one is needed: the
        calls of a step share it in the order of the stream."""
        if name not in self.ws or self.ws[name].numel() < need:
            self.ws[name] = make()
        return self.ws[name]

    def _matmul(self, x, w):
        if isinstance(w, qlm.F8):
            ws = self._workspace("f8", qlm.f8_workspace_bytes(w, x.shape[0]),
                                 lambda: qlm.f8_workspace(w, x.shape[0]))
            return qlm.f8_matmul(qlm.f8_rows(x), w, dtype=x.dtype, ws=ws)
        ws = self._workspace("w4", qlm.w4_workspace_bytes(w, x.shape[0]),
                             lambda: qlm.w4_workspace(w, x.shape[0]))
        return qlm.w4_matmul(x, w, ws=ws)

    def forward(self, x, new):
        """x [batch * new, hidden] through the layers; `new` tokens a sequence."""
        m = self.model
        self.lengths += new
        start = torch.arange(self.batch + 1, dtype=torch.int32, device="cuda") * new
        batch = qlm.KvBatch(self.table, self.lengths, start, self.batch * new, new)
        for cache, (w_qkv, w_out, w_up, w_down) in zip(self.caches, m.layers):
            qkv = self._matmul(x, w_qkv).view(-1, m.heads + 2 * m.kv_heads, m.dim)
            q = qkv[:, :m.heads]
            k, v = qkv[:, m.heads:m.heads + m.kv_heads], qkv[:, m.heads + m.kv_heads:]
            if self.rotary is not None:
                q = qlm.kv_append_rotated(cache, batch, k, v, q, self.rotary,
                                          first_position=self.next)
            else:
                qlm.kv_append(cache, batch, k, v, self.next)
            need = qlm.kv_attention_workspace_bytes(cache, batch, m.heads, True)
            ws = self._workspace("attention", need,
                                 lambda: qlm.kv_attention_workspace(cache, batch, m.heads, True))
            att = qlm.kv_attention(cache, batch, q, weight_decay=1.0, ws=ws)
            x = x + self._matmul(att.view(x.shape[0], -1), w_out)
            x = x + self._matmul(torch.nn.functional.silu(self._matmul(x, w_up)), w_down)
        self.next += new
        self.position += new
        return x

    def restart(self):
        """Every sequence without a token again."""
        self.lengths.zero_()
        self.next.zero_()
        self.position = 0

    def decode(self, x, steps, budget, recent):
        """Steps of one token a sequence, queued without waiting for the GPU; a block that
        is full is followed by a cut to the budget."""
        for _ in range(steps):
            y = self.forward(x, 1)
            if self.position % BLOCK == 0:
                self.evict(budget, recent)
        return y

    def probabilities(self, y):
        return torch.softmax(self._matmul(y, self.model.head).float(), -1)

    def draft(self, tokens, n, gen):
        """n tokens drafted behind tokens [batch], and the probabilities that they were drawn
        from: the model without its layers."""
        one = qlm.KvBatch(self.table, self.lengths)
        drafts, near = [tokens], []
        for _ in range(n):
            near.append(self.probabilities(self.model.words[drafts[-1]]))
            u = torch.rand(self.batch, generator=gen, device="cuda")
            drawn, _, _ = qlm.draft_verify(one, drafts[-1], near[-1], None, u)
            drafts.append(drawn[:, 0])
        near.append(torch.zeros_like(near[0]) if near else None)     # (behind the last: not read)
        return torch.stack(drafts, 1), torch.stack(near, 1) if n else None

    def drafted_step(self, tokens, n, gen):
        """One step over n drafts behind tokens [batch]: the tokens that it gives [batch, n + 1]
        (-1 past their number) and their number [batch].  The cache keeps the accepted ones.
        Attention comes before the verification: the weights by which a later cut chooses hold what
        the refused drafts' rows gave to the slots before them, too."""
        rows, near = self.draft(tokens, n, gen)
        start = torch.arange(self.batch + 1, dtype=torch.int32, device="cuda") * (n + 1)
        first = self.next.clone()
        target = self.probabilities(self.forward(self.model.words[rows.flatten()], n + 1))
        batch = qlm.KvBatch(self.table, self.lengths, start, self.batch * (n + 1), n + 1)
        u = torch.rand(self.batch * (n + 1), generator=gen, device="cuda")
        got, count, _ = qlm.draft_verify(batch, rows.flatten(), target,
                                         None if near is None else near.flatten(0, 1), u,
                                         lengths=self.lengths)
        self.next = first + count
        return got, count

    def drafted(self, tokens, n, steps, budget, recent, gen):
        """Steps over drafts, queued without waiting for the GPU; the number of tokens that they
        give.  Sequences are cut to the budget before they can have grown by a block."""
        if n + 1 > BLOCK:
            raise ValueError("at most %d drafts" % (BLOCK - 1))
        total = torch.zeros((), dtype=torch.int64, device="cuda")
        each = BLOCK // (n + 1)
        for i in range(steps):
            got, count = self.drafted_step(tokens, n, gen)
            tokens = got.gather(1, (count - 1).long()[:, None])[:, 0].contiguous()
            total += count.sum()
            if (i + 1) % each == 0:
                self.evict(budget, recent)
        return total

    def evict(self, budget, recent):
        batch = qlm.KvBatch(self.table, self.lengths)
        need = qlm.kv_evict_workspace_bytes(self.caches[0], batch, budget)
        ws = self._workspace("evict", need,
                             lambda: qlm.kv_evict_workspace(self.caches[0], batch, budget))
        out = torch.empty_like(self.lengths)
        for cache in self.caches:
            qlm.kv_evict(cache, batch, budget, recent, out=out, ws=ws)
        self.lengths.copy_(out)


def measure(model, layers, batch, prompt, budget, recent, steps, memory, drafts=0):
    """The profile's numbers for this model on this GPU: prefill and decode
    seconds, and the tokens that `memory` bytes hold beside the weights."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    inst = Instance(model, layers, batch, max(prompt, budget) + 2 * BLOCK,
                    prompt + (steps + 4) * (drafts + 1) if drafts else 0)
    rnd = lambda n: torch.randn((n, model.hidden), generator=gen, device="cuda",  # noqa: E731
                                dtype=torch.bfloat16)

    def timed(f):
        torch.cuda.synchronize()
        t = time.perf_counter()
        f()
        torch.cuda.synchronize()
        return time.perf_counter() - t

    x = rnd(batch * prompt)
    inst.forward(x, prompt)                        # first use: workspaces, memory
    inst.restart()
    prefill = timed(lambda: inst.forward(x, prompt)) / batch

    y = rnd(batch)

    inst.evict(budget, recent)
    if drafts:
        tokens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        inst.drafted(tokens, drafts, 1, budget, recent, gen)     # first use
        inst.evict(budget, recent)
        given = []
        seconds = timed(lambda: given.append(inst.drafted(tokens, drafts, steps, budget, recent,
                                                          gen)))
        tokens_a_step = int(given[0]) / (batch * steps)
        return {"prefill": prefill, "decode_time": seconds / steps / tokens_a_step,
                "kv_tokens": (memory - model.weight_bytes(layers)) / model.token_bytes(layers),
                "lengths": inst.lengths, "tokens_a_step": tokens_a_step}
    inst.forward(y, 1)
    seconds = timed(lambda: inst.decode(y, steps, budget, recent)) / steps
    assert bool(torch.isfinite(inst.forward(y, 1)).all())
    return {"prefill": prefill, "decode_time": seconds,
            "kv_tokens": (memory - model.weight_bytes(layers)) / model.token_bytes(layers),
            "lengths": inst.lengths, "tokens_a_step": 1.0}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--layers", type=int, default=16)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--inner", type=int, default=16384)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--budget", type=int, default=1024)
    ap.add_argument("--recent", type=int, default=128)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--memory-gb", type=float, default=288.0)
    ap.add_argument("--plans", type=int, default=4096)
    ap.add_argument("--bits", type=int, choices=(4, 8), default=4)
    ap.add_argument("--drafts", type=int, default=0)
    ap.add_argument("--vocab", type=int, default=32000)
    a = ap.parse_args(argv)

    # two models that take turns on the instances of one class: the second of half
    # the layers
    model = Model(a.hidden, a.heads, a.kv_heads, a.dim, a.inner, layers=a.layers, bits=a.bits,
                  vocab=a.vocab if a.drafts else 0)
    layers = [a.layers, max(1, a.layers // 2)]
    got = [measure(model, n, a.batch, a.prompt, a.budget, a.recent, a.steps, a.memory_gb * 1e9,
                   a.drafts) for n in layers]
    for n, g in zip(layers, got):
        print("%2d layers: prefill %.2f ms a prompt of %d, decode step %.3f ms (batch %d), "
              "%.3g tokens of cache" % (n, 1e3 * g["prefill"], a.prompt, 1e3 * g["decode_time"],
                                        a.batch, g["kv_tokens"]), flush=True)
        if a.drafts:
            print("           %d drafts a sequence: a step gives %.2f tokens (seconds are a token's)"
                  % (a.drafts, g["tokens_a_step"]), flush=True)

    problem = workload.make_problem("mixed")
    plans = workload.make_plans(problem, 0, a.plans)
    dpr, dpl = qlm.DeviceProblem(problem), qlm.DevicePlans.from_host(plans)
    one = lambda key: np.array([g[key] for g in got], np.float32)  # noqa: E731
    classes = problem["n_classes"]
    per_class = lambda v: np.tile(v, (classes, 1))  # noqa: E731
    profile = {"prefill": one("prefill"), "decode_time": per_class(one("decode_time")),
               # (the step measured holds a.batch sequences of a.budget tokens; one over the
               # whole memory takes in proportion longer)
               "ineff": per_class(one("kv_tokens") / (a.batch * a.budget)),
               "max_tokens": np.full(2, 1000, np.float32),
               "kv_tokens": per_class(one("kv_tokens")),
               "mean_tokens": np.full(2, a.budget, np.float32)}
    loaded = np.arange(problem["n_instances"]) % problem["n_models"]
    measured, _ = qlm.apply_profile(dpr, profile, inst_model=loaded)
    index, score = qlm.best_plan(measured, dpl)
    print("throughput of an instance: %s tokens/s" %
          ", ".join("%.0f" % t for t in measured.inst_tput.cpu().tolist()[:2]))
    print("best of %d plans: %d, %.1f of %d requests expected to miss their SLO"
          % (a.plans, int(index), float(score), dpr.total_requests), flush=True)
    return {"profile": profile, "best": int(index), "score": float(score), "measured": got}


if __name__ == "__main__":
    main()
