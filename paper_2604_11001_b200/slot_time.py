"""From slots to seconds: what a slot of the simulated system takes on the GPU, for one attention layer.

The simulator's clock is the slot, in which every active request generates one token.  This module runs such slots on a
real paged cache (``kvcache``): active sets drawn from a preset's length laws at the KV usages U_t that a simulated run
of the preset goes through, one append and one attend per slot, timed on the device; then a line

    microseconds(U) = a + b U

through the times, and with it the simulated run's results in seconds per layer instead of slots: the run's own trace gives
every slot's U_t and so its time (a slot without requests takes that of an empty one, a), its log every request's first and last
slot, whose times add up to its latency.  In a slot's time are the new tokens of its requests, not the prompts of those that
begin in it: nothing here attends over a prompt.  With ``--budget`` each request's cache is also cut to that many tokens by accumulated attention
weight, whenever it has grown ``SLACK`` tokens past it: the eviction of tokens that the slotted model, which evicts whole
requests, has no form of.  The requests of a slot stay those of the simulated run (admission counts whole requests, and U is
their usage); what the budget changes is what they hold on the GPU, and the time of a slot, to which the cuts add.

    python -m paper_2604_11001_b200.slot_time [--preset 2] [--slots 2000] [--cache e4m3] [--budget 256]
"""
from __future__ import annotations

import argparse
from typing import List, Optional

import numpy as np

from . import workloads as wl

PRESETS = {k: f for k, f in wl.PRESETS.items() if k != 3}   # (preset 3 is a sweep of 4 096 groups)
PAGE = 16
SLACK = 64          # tokens by which a request outgrows its budget before it is cut
FIRST = 4           # oldest tokens that are always kept


def _draw(table: wl.Table, rng) -> int:
    values, p = wl.table_pmf(table)
    return int(values[np.searchsorted(np.cumsum(p), rng.random(), side="right").clip(max=len(values) - 1)])


def active_set(cfg: wl.SimConfig, usage: int, rng, limit: Optional[int] = None) -> List[int]:
    """Lengths of requests that hold `usage` tokens together: classes and lengths from the preset's laws, generated
    tokens as in a slot picked at random (an output of o tokens is met o times as often, at a uniform point of it).
    At most ``cfg.Acap`` requests.  ``limit`` (a token budget) then cuts every one: the requests stay the same."""
    lengths: List[int] = []
    held = 0
    longest = [t.vmax for t in cfg.decode]
    while held < usage and len(lengths) < cfg.Acap:
        k = _draw(cfg.class_law, rng)
        prompt, out = _draw(cfg.prompt[k], rng), _draw(cfg.decode[k], rng)
        if rng.random() * max(longest) > out:
            continue
        n = min(prompt + int(rng.integers(0, out)), usage - held)
        lengths.append(n)
        held += n
    return lengths if limit is None else [min(n, limit) for n in lengths]


class Layer:
    """One layer's cache with room for `lengths` and for what they grow to in `spare` slots, and the slots on it."""

    def __init__(self, lengths, heads=64, kv_heads=8, head_dim=128, cache="bf16", budget=None, spare=256, device="cuda:0", seed=0):
        import torch

        from .kvcache import PagedKV
        self.torch, self.budget, self.device = torch, budget, torch.device(device)
        self.spare_slots = spare
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.dtype = torch.float16 if cache == "f16" else torch.bfloat16
        store = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[cache]
        self.generator = torch.Generator(device=self.device)
        self.generator.manual_seed(seed)
        grown = max(lengths) + spare + 1 if budget is None else budget + SLACK   # (one more: time() after the last)
        self.columns = -(-max(grown, max(lengths) + 1) // PAGE)
        pages = len(lengths) * self.columns * (1 if budget is None else 2)
        self.cache = PagedKV.allocate(pages, PAGE, kv_heads, head_dim, store, weight=budget is not None, device=self.device)
        order = torch.randperm(pages, generator=self.generator, device=self.device).to(torch.int32)
        n = len(lengths)
        self.table = order[:n * self.columns].view(n, self.columns).contiguous()
        self.spare = None if budget is None else order[n * self.columns:].view(n, self.columns).contiguous()
        self.lengths = torch.zeros(n, dtype=torch.int32, device=self.device)
        self.positions = torch.zeros(n, dtype=torch.int32, device=self.device)   # of the next token; cut requests go on counting
        angle = torch.arange(max(lengths) + spare + 1, device=self.device, dtype=torch.float64)[:, None] \
            * 10000.0 ** (-torch.arange(0, head_dim, 2, device=self.device, dtype=torch.float64) / head_dim)
        self.rope = torch.cat((angle.cos(), angle.sin()), 1).float()
        self.norm = torch.ones(head_dim, dtype=self.dtype, device=self.device)
        self._prompts(lengths)

    def _rows(self, n, heads):
        return self.torch.randn(n, heads, self.head_dim, generator=self.generator, device=self.device).to(self.dtype)

    def _slots(self, requests, tokens):
        pages = self.table[requests, tokens // PAGE].long()
        return pages * PAGE + (tokens % PAGE).long()

    def _prompts(self, lengths):
        """Load the requests' prompts, at most 16 384 tokens at a time."""
        torch = self.torch
        request = torch.repeat_interleave(torch.arange(len(lengths), device=self.device),
                                          torch.tensor(lengths, device=self.device))
        token = torch.cat([torch.arange(n, device=self.device) for n in lengths])
        for at in range(0, token.numel(), 16384):
            r, t = request[at:at + 16384], token[at:at + 16384]
            self.cache.append(None, self._rows(t.numel(), self.kv_heads), self._rows(t.numel(), self.kv_heads),
                              t.to(torch.int32), self._slots(r, t), rope=self.rope, k_norm=self.norm)
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device=self.device)
        self.positions = self.lengths.clone()

    def step(self, q, k, v, slots):
        """What every slot does: one token per request goes in, one query per request reads its tokens."""
        q = self.cache.append(q, k, v, self.positions, slots, rope=self.rope, q_norm=self.norm, k_norm=self.norm)
        return self.cache.attend(q, self.table, self.lengths, add_weight=self.budget is not None)

    def grow(self):
        """One whole slot: a new token per request, then the cut of those that have outgrown their budget."""
        torch = self.torch
        if self.spare_slots == 0:
            raise ValueError("the layer has no room (pages, positions) for another slot: make it with more `spare`")
        self.spare_slots -= 1
        n = self.lengths.numel()
        slots = self._slots(torch.arange(n, device=self.device), self.lengths)
        self.lengths += 1
        out = self.step(self._rows(n, self.heads), self._rows(n, self.kv_heads), self._rows(n, self.kv_heads), slots)
        self.positions += 1
        if self.budget is not None:
            over = (self.lengths >= self.budget + SLACK).nonzero()[:, 0]
            if over.numel():
                old, new = self.table[over].contiguous(), self.spare[over].contiguous()
                kept, _ = self._cut(old, self.lengths[over].contiguous(), new)
                self.lengths[over] = kept
                self.table[over], self.spare[over] = new, old
        return out

    def _cut(self, old, lengths, new):
        budget = self.torch.full_like(lengths, self.budget)
        return self.cache.evict(old, lengths, budget, new, max_budget=self.budget, recent=self.budget // 4, first=FIRST)

    def _timed(self, call, repeats):
        """Microseconds of a call (median, on the device), the L2 cache filled with other data before each."""
        torch = self.torch
        times = []
        with torch.cuda.device(self.device):
            flush = torch.empty(64 << 20, dtype=torch.float32, device=self.device)   # twice the L2 cache
            for i in range(repeats + 3):
                flush.sum()
                a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                a.record()
                call()
                b.record()
                b.synchronize()
                if i >= 3:
                    times.append(a.elapsed_time(b) * 1e3)
        self.cache.check()
        return float(np.median(times))

    def time(self, repeats=20):
        """Microseconds of the next slot.  The layer is left as it was: the slot's tokens lie behind its requests' last ones, and
        the weights are put back."""
        torch = self.torch
        n = self.lengths.numel()
        inputs = (self._rows(n, self.heads), self._rows(n, self.kv_heads), self._rows(n, self.kv_heads),
                  self._slots(torch.arange(n, device=self.device), self.lengths))
        weight = None if self.budget is None else self.cache.weight.clone()
        self.lengths += 1
        us = self._timed(lambda: self.step(*inputs), repeats)
        self.lengths -= 1
        if weight is not None:
            self.cache.weight.copy_(weight)
        return us

    def time_cuts(self, repeats=20):
        """Microseconds that cuts add to a slot on average.  A request past its budget is cut once in SLACK slots, so `due` of them
        are in a slot: one call for these, or, where they are less than one, a call for one in so many slots.  (The rows
        move to the pages that wait for the next cut; the layer is left as it was.)"""
        over = (self.lengths >= self.budget).nonzero()[:, 0]
        due = over.numel() / SLACK
        if due == 0:
            return 0.0
        over = over[:max(1, round(due))]
        old, new = self.table[over].contiguous(), self.spare[over].contiguous()
        lengths = self.torch.full((over.numel(),), self.budget + SLACK, dtype=self.torch.int32, device=self.device)
        return min(1.0, due) * self._timed(lambda: self._cut(old, lengths, new), repeats)


def latency_seconds(seconds, done, latency):
    """Seconds from the first to the last slot of requests that completed in slot `done` (1, 2, ..) after `latency` slots, that one
    and the first included; `seconds` of every slot."""
    clock = np.concatenate(([0.0], np.cumsum(seconds)))
    return clock[done] - clock[done - latency]


def run(preset: int = 2, slots: int = 2000, replicas: int = 16, points: int = 6, grow: int = 0, budget: Optional[int] = None,
        heads: int = 64, kv_heads: int = 8, head_dim: int = 128, cache: str = "bf16", device: str = "cuda:0", seed: int = 0) -> dict:
    """Simulate the preset, time slots at usages its trace goes through, and turn the run's slots into seconds."""
    from . import binding as fb
    cfg = PRESETS[preset](replicas=replicas, T=slots)
    arrivals = max(t.vmax for a in cfg.arrivals for t in a.count)
    cfg = cfg.with_(trace_stride=1, complog_cap=slots * arrivals)   # (no more than that can complete)
    sim = fb.Simulation(cfg, device=device)
    sim.run(slots)
    counters, summary = sim.stats()
    usage = sim.trace()[:, :, 0].cpu().numpy()   # [replicas of all groups, slots]
    logged = counters[:, fb.COUNTER_NAMES.index("n_logged")]
    log = sim.complog()[:, :max(1, int(logged.max()))].cpu().numpy()
    sim.close()
    rng, since_cut = np.random.default_rng(seed), np.random.default_rng([seed, 1])   # (the sets do not depend on the budget)
    busy = usage[usage > 0]
    rows = []
    for u in np.unique(np.quantile(busy, np.linspace(0.05, 1.0, points)).astype(int)):
        whole = active_set(cfg, int(u), rng)
        # with a budget: the same requests, each that has outgrown it somewhere between two cuts
        held = whole if budget is None else [n if n < budget else budget + int(since_cut.integers(0, SLACK)) for n in whole]
        layer = Layer(held, heads, kv_heads, head_dim, cache, budget, spare=grow, device=device, seed=seed)
        cuts = 0.0 if budget is None else layer.time_cuts()
        us = layer.time() + cuts
        for _ in range(grow):
            layer.grow()
        layer.cache.check()
        rows.append(dict(usage=int(sum(whole)), requests=len(whole), longest=max(whole) if budget is None else min(max(whole), budget),
                         held=int(sum(held)), us=us, cuts_us=cuts))
        del layer
    x = np.array([[1.0, r["usage"]] for r in rows])
    a, b = np.linalg.lstsq(x, np.array([r["us"] for r in rows]), rcond=None)[0] if len(rows) > 1 else (rows[0]["us"], 0.0)
    seconds = (a + b * usage) * 1e-6   # of every slot of every replica
    out = dict(preset=cfg.name, rows=rows, a_us=float(a), b_us=float(b), groups=[])
    start = 0
    for g, s in zip(cfg.groups, summary):
        mine = range(start, start + g.n_replicas)
        start += g.n_replicas
        slot = float(seconds[mine].mean())
        waits = np.concatenate([latency_seconds(seconds[r], *log[r, :logged[r]].T) for r in mine])
        out["groups"].append(dict(policy=g.policy, slot_us=slot * 1e6, mean_latency_slots=s["mean_latency"],
                                  mean_latency_ms=float(waits.mean()) * 1e3 if waits.size else float("nan"),
                                  tokens_per_second=s["token_throughput"] / slot))
    return out


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--preset", type=int, default=2, choices=sorted(PRESETS))
    ap.add_argument("--slots", type=int, default=2000)
    ap.add_argument("--replicas", type=int, default=16)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--cache", default="bf16", choices=("bf16", "f16", "e4m3"))
    ap.add_argument("--budget", type=int, default=None, help="tokens a request's cache is cut to")
    ap.add_argument("--grow", type=int, default=0, help="slots to run on from each timed set, cuts among them")
    args = ap.parse_args()
    got = run(args.preset, args.slots, args.replicas, grow=args.grow, budget=args.budget, heads=args.heads, kv_heads=args.kv_heads,
              head_dim=args.head_dim, cache=args.cache)
    print("%s, one layer, %d heads on %d of %d, %s cache (no prompts in the times)" % (got["preset"], args.heads, args.kv_heads, args.head_dim, args.cache))
    print("%10s %10s %10s %10s %12s %12s" % ("tokens", "requests", "longest", "held", "us per slot", "of it cuts"))
    for r in got["rows"]:
        print("%10d %10d %10d %10d %12.2f %12.2f" % (r["usage"], r["requests"], r["longest"], r["held"], r["us"], r["cuts_us"]))
    print("us(U) = %.2f + %.6f U" % (got["a_us"], got["b_us"]))
    for g in got["groups"]:
        print("policy %d: %.2f us a slot, mean latency %.1f slots = %.3f ms a layer, %.0f tokens/s a layer" % (
            g["policy"], g["slot_us"], g["mean_latency_slots"], g["mean_latency_ms"], g["tokens_per_second"]))


if __name__ == "__main__":
    main()
