"""An offline-inference job that the price loop resizes while it decodes.

Eight jobs share a cluster; a job's configurations are batch sizes, each with
the compute and the cache memory it takes.  The price loop picks one for every
job.  Job 0 then runs in the paged 8-bit cache: prompts enter, each is forked
to fill the batch, tokens are decoded, and when the cluster has less memory the
job ends sequences, compacts its pages into the smaller budget, gives the rest of
the pool back and goes on.
The layers are projections with random weights around the cache's operators.

    python examples/elastic_inference.py [--steps N]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_07971_amd as esp  # noqa: E402
from paper_2608_07971_amd import kv  # noqa: E402
import workloads  # noqa: E402

BATCHES = [4, 8, 16, 32]
JOBS, LAYERS, KV_HEADS, GROUP, DIM, PAGE = 8, 2, 2, 4, 64, 16
PROMPT, LONGEST = 60, 256
PAGES_A_SEQUENCE = LONGEST // PAGE


def cluster(memory: float) -> workloads.Instance:
    """The jobs' table: resources compute and memory, in batches' worth of sequences."""
    batch = np.array(BATCHES, dtype=np.float64)
    weight = 1.0 + 0.05 * np.arange(JOBS)[::-1]                       # job 0 counts most
    utility = (weight[:, None] * np.log2(1.0 + batch) / 5.0).reshape(1, -1).astype(np.float32)
    demand = np.tile(np.stack([batch / 32.0, batch / 32.0], -1), (JOBS, 1))[None].astype(np.float32)
    return workloads.Instance(name="elastic", seed=0, offsets=np.arange(JOBS + 1, dtype=np.int64) * len(BATCHES), utility=utility,
                              demand=demand, capacity=np.array([[JOBS, memory]], dtype=np.float64), eta0=np.array([0.02]),
                              rule=workloads.STEP_INV_SQRT, lam0=np.zeros((1, 2)), iters=200)


def batch_of_job(memory: float) -> int:
    """The batch size of job 0 that the prices for this much memory lead to."""
    solver = esp.Solver(cluster(memory))
    choice = solver.solve(solver.prices(np.zeros((1, 2))), 200)["choice"]
    k = int(choice[0, 0])
    assert solver.device_status() == 0
    solver.close()
    return BATCHES[k]


class Job:
    """The job's layers, its cache and the hidden state of every sequence's last token."""

    def __init__(self, batch: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        heads, self.hidden = KV_HEADS * GROUP, KV_HEADS * GROUP * DIM

        def weights(*shape):
            return (torch.randn(shape, device="cuda", generator=g) / math.sqrt(shape[0])).half()

        self.project = [weights(self.hidden, (heads + 2 * KV_HEADS) * DIM) for _ in range(LAYERS)]
        self.back = [weights(heads * DIM, self.hidden) for _ in range(LAYERS)]
        self.rope = kv.Rope(DIM, scaling="parts", factor=4.0, context=64)
        self.cache = kv.PagedCache(batch * PAGES_A_SEQUENCE, PAGE, KV_HEADS, DIM, max(BATCHES), PAGES_A_SEQUENCE, layers=LAYERS)
        self.budget, self.g = self.cache.pages, g
        self.lengths = [0] * max(BATCHES)                            # the host's copy: it chose them
        self.state = torch.zeros(max(BATCHES), self.hidden, dtype=torch.float16, device="cuda")

    def _ints(self, x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    def forward(self, seqs, counts, x):
        """New tokens x of these sequences through the layers; the last token's state of each is kept."""
        for s, n in zip(seqs, counts):
            self.lengths[s] += n
        self.cache.resize(self._ints(self.lengths))
        offsets, rows = self._ints(np.concatenate([[0], np.cumsum(counts)])), self._ints(seqs)
        heads, most, longest = KV_HEADS * GROUP, max(counts), max(self.lengths[s] for s in seqs)
        for layer in range(LAYERS):
            q, k, v = torch.matmul(x, self.project[layer]).view(len(x), -1, DIM).split([heads, KV_HEADS, KV_HEADS], dim=1)
            q = self.cache.append(layer, k, v, offsets, rope=self.rope, q=q, seqs=rows)
            out, lse = self.cache.attend(layer, q, offsets, seqs=rows, max_new=most, max_length=longest)
            x = x + torch.matmul(out.reshape(len(x), -1), self.back[layer])
            x = x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).half()
        self.state[rows.long()] = x[offsets[1:].long() - 1]
        return layer, q, offsets, rows, out, lse

    def live(self):
        return [s for s, n in enumerate(self.lengths) if n]

    def prompts(self, n: int):
        """n prompts of unequal lengths."""
        counts = [PROMPT - 7 * (i % 5) for i in range(n)]
        x = torch.randn(sum(counts), self.hidden, device="cuda", generator=self.g).half()
        return self.forward(list(range(n)), counts, x)

    def fill(self, batch: int):
        """Every live sequence goes on in as many places as the batch has for it."""
        live, free = self.live(), [s for s, n in enumerate(self.lengths) if not n]
        children = free[:batch - len(live)]
        parents = [live[i % len(live)] for i in range(len(children))]
        self.cache.fork(self._ints(parents), self._ints(children))
        for p, c in zip(parents, children):
            self.lengths[c] = self.lengths[p]
            self.state[c] = self.state[p]
        noise = torch.randn(self.state.shape, device="cuda", generator=self.g).half()
        self.state += 0.1 * noise                                    # so that the branches differ

    def decode(self, steps: int):
        for _ in range(steps):
            seqs = self.live()
            last = self.forward(seqs, [1] * len(seqs), self.state[self._ints(seqs).long()])
        return last

    def shrink(self, batch: int) -> int:
        """Ends the sequences beyond the batch, moves the others' pages into the smaller budget and goes on in a pool of
        that size; pages given back."""
        for s in self.live()[batch:]:
            self.lengths[s] = 0
        self.cache.resize(self._ints(self.lengths))
        before, self.budget = self.budget, min(self.budget, batch * PAGES_A_SEQUENCE)
        table, refs, _ = self.cache.compact(self.budget)
        self.cache.install(table, refs)
        if self.cache.device_status():
            raise RuntimeError("the sequences left do not fit the budget")
        c, n = self.cache, self.budget
        self.cache = kv.PagedCache.adopt(*(t[:n].clone() for t in (c.k, c.v, c.scale)), c.table, c.lengths, c.refs[:n].clone())
        return before - self.budget

    def error(self, step) -> float:
        """Largest difference of a step's attention from 64 bits on what the cache holds, relative to the values."""
        layer, q, offsets, rows, out, _ = step
        seqs, worst = rows.tolist(), 0.0
        for i, s in enumerate(seqs):
            n = self.lengths[s]
            k, v = self.cache.gather(layer, self._ints([0]), self._ints([0, n]), n, dtype=torch.float16, seqs=self._ints([s]))
            at = int(offsets[i + 1]) - 1
            for h in range(KV_HEADS * GROUP):
                kk, vv = (t[:, h // GROUP].cpu().double() for t in (k, v))
                want = torch.softmax(kk @ q[at, h].cpu().double() / math.sqrt(DIM), 0) @ vv
                worst = max(worst, float((out[at, h].cpu().double() - want).abs().max() / vv.abs().max()))
        return worst


def main(steps: int = 24) -> dict:
    wide, narrow = batch_of_job(JOBS), batch_of_job(JOBS / 5)
    job = Job(wide)
    job.prompts(min(4, wide))
    job.fill(wide)
    first = job.error(job.decode(steps))
    freed = job.shrink(min(narrow, wide))
    highest = int(job.cache.table.max())
    second = job.error(job.decode(steps))
    return dict(batches=(wide, narrow), pages=(wide * PAGES_A_SEQUENCE, job.budget), freed=freed, bytes=freed * job.cache.page_bytes,
                highest=highest,
                lengths=[n for n in job.lengths if n], errors=(first, second), status=job.cache.device_status())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=24, help="tokens decoded before and after the change of budget")
    r = main(p.parse_args().steps)
    print(f"batch {r['batches'][0]} -> {r['batches'][1]}, pages {r['pages'][0]} -> {r['pages'][1]} ({r['freed']} of {r['bytes']:,} bytes given back, "
          f"highest page in use {r['highest']})")
    print(f"sequences of {r['lengths']} tokens; attention within {max(r['errors']):.1e} of 64 bits; status {r['status']}")
