"""A decode loop on the pool, the block table and the operators on the device cache, as a serving engine would run it.

    python -m paper_2601_20309_b200.decode [--layers L] [--requests R] [--prompt P] [--steps S] [--keep K] [--slack D] [--norms]
        R requests with prompts of P tokens on the 8B shape's heads, S tokens each: per step and layer one kv_append and one
        kv_attend; whenever a request holds K + D tokens, kv_evict takes it back to K in all layers and the block table
        gets its blocks back; every 16 steps half of the requests are preempted to host memory and resumed.  Reports
        the step's device time, the blocks held, the blocks a preemption moves and their MB, with and without eviction, with the cache
        in 16 bits and in 4.  --norms: queries and keys are normed per head.  (Projections and the rest of a model are left
        out: q, k and v are random.)
"""
from __future__ import annotations

import argparse
import contextlib
import sys

from . import binding as B


class Decoder:
    """Requests in `places` rows of a batch of fixed size, of up to max_tokens tokens each; a row without a request on the GPU is idle
    (length 0).  The cache is held in 16 or in 4 `bits`.  q_norm, k_norm: weights of norms per head in front of the rotation, [layers, head_dim] or
    [layers, heads, head_dim] (``kv_append``), with norm_eps.  Weights and ages of the slots are kept per layer and place; block tables and lengths go to the device once per call.
    Kernels and copies run on the stream that is current when the decoder is made, in order with the stream a method is called under."""

    def __init__(self, num_layers, block_size, q_heads, kv_heads, head_dim, num_gpu_blocks, num_host_blocks, places, max_tokens, *, keep=0,
                 slack=0, recent=0, sink=0, sections=None, theta=10000.0, device=0, bits=16, q_norm=None, k_norm=None, norm_eps=1e-6):
        import torch
        if bits not in (16, 4):
            raise ValueError("the cache is held in 16 or 4 bits")
        self.torch, self.device = torch, torch.device("cuda", device)
        self.layers, self.bs, self.q_heads, self.kv_heads, self.dim = num_layers, block_size, q_heads, kv_heads, head_dim
        self.keep, self.slack, self.recent, self.sink = keep, slack, recent, sink
        self.q_norm, self.k_norm, self.norm_eps = q_norm, k_norm, norm_eps
        dtype = "bf16" if bits == 16 else "bf16_q4"
        units = B.kv_cache_row_units(dtype, head_dim)       # of a row: its elements, or its codes and words
        if not units:
            raise ValueError(f"no cache for heads of {head_dim}")
        self.store = torch.zeros(num_layers, 2, num_gpu_blocks, block_size, kv_heads, units, dtype=torch.bfloat16, device=self.device)
        self.pool = B.KVPool(num_layers, block_size, kv_heads, units, num_gpu_blocks, num_host_blocks, self.store.data_ptr(), device_id=device)
        self.table = B.KVTable(self.pool)
        self.own = torch.cuda.current_stream(self.device)
        self.stream = self.own.cuda_stream
        self.ops = B.KVOps(device, self.stream)
        self.cache = self.pool.kv_pool_cache(dtype, head_dim)
        half = head_dim // 2
        self.inv_freq = (theta ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(self.device)
        self.axis_of = [a for a, n in enumerate(sections) for _ in range(n)] if sections else [0] * half
        self.max_tokens, self.width = max_tokens, -(-max_tokens // block_size)
        self.weights = torch.zeros(num_layers, places, kv_heads, max_tokens, device=self.device)
        self.order = torch.zeros(num_layers, places, kv_heads, max_tokens, dtype=torch.int32, device=self.device)
        self.place_of: dict = {}                # request -> row, whether on the GPU or not
        self.held = [0] * places                # tokens in the cache, per row
        self.seen = [0] * places                # tokens there ever were
        self.running = [False] * places
        self.out = torch.zeros(num_layers, places, q_heads, head_dim, dtype=torch.bfloat16, device=self.device)
        self.turned = torch.zeros(places, q_heads, head_dim, dtype=torch.bfloat16, device=self.device)

    def _norms(self, layer, q=True):
        """What a layer's ``kv_append`` gets for its norms."""
        return {"q_norm": self.q_norm[layer] if q and self.q_norm is not None else None,
                "k_norm": self.k_norm[layer] if self.k_norm is not None else None, "norm_eps": self.norm_eps}

    def close(self):
        self.torch.cuda.synchronize(self.device)
        self.ops.destroy()
        self.table.destroy()
        self.pool.destroy()

    @contextlib.contextmanager
    def _on_own_stream(self):
        """All work of a call goes to the stream the decoder was made on: after what the caller's current stream holds so far (the
        call's inputs), and before what comes next there (who reads the results or gives the inputs' memory to something else)."""
        caller = self.torch.cuda.current_stream(self.device)
        if caller == self.own:
            yield
            return
        self.own.wait_stream(caller)
        try:
            with self.torch.cuda.stream(self.own):
                yield
        finally:
            caller.wait_stream(self.own)

    def _upload(self, rows=None):
        """Block tables and lengths of the given rows (others count as idle)."""
        t = self.torch
        tables, lens = t.full((len(self.held), self.width), -1, dtype=t.int32), t.zeros(len(self.held), dtype=t.int32)
        for req, row in self.place_of.items():
            if self.running[row] and (rows is None or row in rows):
                ids = self.table.kv_req_blocks(req)[0]
                tables[row, :len(ids)] = t.from_numpy(ids)
                lens[row] = self.held[row]
        return tables.to(self.device), lens.to(self.device)

    def _check(self, qkv, positions, n):
        """Tensors of n tokens, before anything is booked for them."""
        t, shape = self.torch, (self.layers, n, self.q_heads + 2 * self.kv_heads, self.dim)
        if tuple(qkv.shape) != shape or qkv.dtype != t.bfloat16 or qkv.device != self.device:
            raise ValueError(f"qkv must be bf16 {shape} on {self.device}")
        if positions.dim() != 2 or positions.shape[0] <= max(self.axis_of) or positions.shape[1] != n or positions.dtype != t.int32 \
                or positions.device != self.device:
            raise ValueError(f"positions must be int32 ({max(self.axis_of) + 1} or more, {n}) on {self.device}")

    def add(self, req, qkv, positions):
        """A request with its prompt: qkv [layers, tokens, q_heads + 2 kv_heads, dim], positions int32 [axes, tokens].  What does not
        fit (no place, more than max_tokens tokens: ``ValueError``; no blocks: ``KVError``) leaves everything as it was."""
        t, h, k = self.torch, self.q_heads, self.kv_heads
        n = qkv.shape[1]
        self._check(qkv, positions, n)
        if n > self.max_tokens:
            raise ValueError(f"a request of {n} tokens, max_tokens is {self.max_tokens}")
        row = next((r for r in range(len(self.held)) if r not in self.place_of.values()), None)
        if row is None:
            raise ValueError(f"all {len(self.held)} places are taken")
        self.table.kv_req_add(req, n)
        try:
            with self._on_own_stream():
                self.pool.kv_stream_wait(self.stream)
                self.place_of[req], self.held[row], self.seen[row], self.running[row] = row, n, n, True
                tables, lens = self._upload({row})
                starts = t.tensor([0, n], dtype=t.int32, device=self.device)
                numbers = t.arange(n, dtype=t.int32, device=self.device)
                one = slice(row, row + 1)
                for layer in range(self.layers):
                    x = qkv[layer]
                    self.ops.kv_append(self.cache, layer, None, x[:, h:h + k], x[:, h + k:], tables[one], lens[one], positions=positions,
                                       inv_freq=self.inv_freq, axis_of=self.axis_of, seq_starts=starts, weights=self.weights[layer, one],
                                       order=self.order[layer, one], token_order=numbers, **self._norms(layer, q=False))
        except BaseException:
            self.ops.kv_ops_sync(check=False)   # kernels of earlier layers may still write the blocks that go back
            self.table.kv_req_finish(req, check=False)
            self.place_of.pop(req, None)
            self.held[row], self.seen[row], self.running[row] = 0, 0, False
            raise

    def step(self, qkv, positions):
        """One token for every running row: qkv [layers, places, q_heads + 2 kv_heads, dim], positions int32 [axes, places].
        Returns the attention's outputs [layers, places, q_heads, dim] (idle rows: zeros), in a buffer that the next step overwrites.
        A step that a running row has no room for (it holds max_tokens: ``ValueError``), or that there are not enough blocks for
        (``KVError`` with KV_ERR_NOMEM: preempt something and repeat it), changes nothing."""
        t, h, k = self.torch, self.q_heads, self.kv_heads
        self._check(qkv, positions, len(self.held))
        rows = [(req, row) for req, row in self.place_of.items() if self.running[row]]
        for req, row in rows:
            if self.held[row] >= self.max_tokens:
                raise ValueError(f"request {req} holds max_tokens = {self.max_tokens} tokens")
        need, free = sum(self.held[row] % self.bs == 0 for _, row in rows), self.table.kv_table_get_stats()["free_gpu_blocks"]
        if need > free:
            raise B.KVError(B.KV_ERR_NOMEM, f"the step needs {need} blocks, {free} are free")
        done = []
        try:
            for req, row in rows:
                self.table.kv_req_append(req, 1)
                done.append((req, row))
                self.held[row] += 1
                self.seen[row] += 1
            with self._on_own_stream():
                tables, lens = self._upload()
                numbers = t.tensor([max(0, s - 1) for s in self.seen], dtype=t.int32, device=self.device)
                longest = max(self.held)
                for layer in range(self.layers):
                    x = qkv[layer]
                    self.ops.kv_append(self.cache, layer, x[:, :h], x[:, h:h + k], x[:, h + k:], tables, lens, positions=positions,
                                       inv_freq=self.inv_freq, axis_of=self.axis_of, q_out=self.turned, weights=self.weights[layer],
                                       order=self.order[layer], token_order=numbers, **self._norms(layer))
                    self.ops.kv_attend(self.cache, layer, self.turned, tables, lens, longest, out=self.out[layer],
                                       weights_in=self.weights[layer], weights_out=self.weights[layer])
        except BaseException:               # no row keeps a token that was not written in every layer
            self.ops.kv_ops_sync(check=False)
            for req, row in done:
                self.held[row] -= 1
                self.seen[row] -= 1
                self.table.kv_req_shrink(req, self.held[row], check=False)
            raise
        full = {row for row in range(len(self.held)) if self.running[row] and self.keep and self.held[row] >= self.keep + self.slack}
        if full:
            with self._on_own_stream():
                self._evict(full)
        return self.out

    def _evict(self, rows):
        t = self.torch
        tables, lens = self._upload(rows)
        seen = t.tensor(self.seen, dtype=t.int32, device=self.device)
        self.pool.kv_stream_wait(self.stream)   # copies in flight may still read the rows
        self.ops.kv_evict(self.cache, tables, lens, max(self.held[r] for r in rows), keep=self.keep, recent=self.recent, sink=self.sink,
                          weights=self.weights, order=self.order, seen=seen)
        self.ops.kv_ops_sync()                  # the blocks go back to the table: nothing may still use them
        for req, row in self.place_of.items():
            if row in rows:
                self.held[row] = self.keep
                self.table.kv_req_shrink(req, self.keep)

    def rotate(self, preempt, resume):
        """Whole requests out to host memory and back in."""
        self.ops.kv_ops_sync()
        self.table.kv_req_rotate(preempt, resume)
        for reqs, on in ((preempt, False), (resume, True)):
            for req in reqs:
                self.running[self.place_of[req]] = on
        self.pool.kv_stream_wait(self.stream)


def run(layers, requests, prompt, steps, keep, slack, seed=1, bits=16, norms=False):
    """The command's loop; a dict of what it measured."""
    import torch
    weights = torch.ones(layers, 128, dtype=torch.bfloat16, device="cuda") if norms else None
    shape = dict(block_size=16, q_heads=32, kv_heads=8, head_dim=128)
    most = (max(prompt, keep) + slack + 1) if keep else prompt + steps
    blocks = requests * (-(-max(most, prompt) // 16) + 2)
    d = Decoder(layers, *shape.values(), blocks, 2 * blocks, requests, max(most, prompt + 1), keep=keep, slack=slack, recent=keep // 8,
                sink=4, sections=(16, 24, 24), bits=bits, q_norm=weights, k_norm=weights)
    g = torch.Generator(device="cuda").manual_seed(seed)
    heads = shape["q_heads"] + 2 * shape["kv_heads"]
    for r in range(requests):
        x = torch.randn(1, prompt, heads, 128, generator=g, device="cuda").to(torch.bfloat16).expand(layers, -1, -1, -1)
        d.add(r, x, torch.arange(prompt, dtype=torch.int32, device="cuda").expand(3, -1).contiguous())
    x = torch.randn(1, requests, heads, 128, generator=g, device="cuda").to(torch.bfloat16).expand(layers, -1, -1, -1)
    begin, end = torch.cuda.Event(True), torch.cuda.Event(True)
    ms, moved = [], []
    for s in range(steps):
        begin.record()
        d.step(x, torch.full((3, requests), prompt + s, dtype=torch.int32, device="cuda"))
        end.record()
        end.synchronize()
        ms.append(begin.elapsed_time(end))
        if s % 16 == 15:
            half = list(range(requests // 2))
            before = d.table.kv_table_get_stats()["preempt_blocks_moved"]
            d.rotate(half, [])
            d.pool.kv_sync()
            moved.append(d.table.kv_table_get_stats()["preempt_blocks_moved"] - before)
            d.rotate([], half)
    held = d.table.kv_table_get_stats()["free_gpu_blocks"]
    ms.sort()
    block_mb = 2 * layers * 16 * 8 * B.kv_cache_row_units("bf16" if bits == 16 else "bf16_q4", 128) * 2 / 1e6
    res = {"step_ms_median": round(ms[len(ms) // 2], 3), "blocks_held": blocks - held, "blocks_moved_per_preemption": moved,
           "mb_moved_per_preemption": [round(n * block_mb, 1) for n in moved]}
    d.close()
    return res


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=32)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--keep", type=int, default=1024)
    ap.add_argument("--slack", type=int, default=128)
    ap.add_argument("--norms", action="store_true")
    a = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        sys.exit("decode needs a CUDA device")
    for bits in (16, 4):
        print(f"{bits:2} bits, whole cache  ", run(a.layers, a.requests, a.prompt, a.steps, 0, 0, bits=bits, norms=a.norms))
        print(f"{bits:2} bits, with eviction", run(a.layers, a.requests, a.prompt, a.steps, a.keep, a.slack, bits=bits, norms=a.norms))


if __name__ == "__main__":
    main()
