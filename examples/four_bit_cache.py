"""A serving loop over a 4-bit cache: prompts, several samples of each, drafts that are accepted or not, eviction.

    python examples/four_bit_cache.py [--samples 4] [--steps 32]

Every request's K and V of one layer are in a pool of 4-bit rows (0.266 of the bytes of bf16):

  prompt   ellm_kv_append quantises the prompt's rows; ellm_kv_read gives the rows as the cache holds them, which is what
           the prompt's own attention should see;
  fork     ellm_kv_copy makes the prompt the beginning of every sample;
  step     the drafts' rows are appended, some are accepted and ellm_kv_compact keeps those; ellm_kv_append_decode then
           writes the next token and attends over everything;
  evict    a request over its budget keeps its first tokens and the newest ones; ELLM_COMPACT_UNMAP gives back the
           chunks that have become empty.

The rows are random: nothing here is a model.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2506_15155_amd as E  # noqa: E402

N_KV, GROUP, DIM = 8, 4, 128
CHUNK = 128 << 10
FIRST = 4                   # tokens that eviction never takes


class Loop:
    def __init__(self, prompts, samples, budget, seed=0):
        self.rng = np.random.default_rng(seed)
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.samples, self.budget = samples, budget
        n = len(prompts) * (1 + samples)
        most = max(budget, max(prompts)) + 64
        probe = E.ellm_pool_create(None, None, CHUNK, N_KV * GROUP, N_KV, DIM, 1, 1, flags=E.ELLM_POOL_METADATA_ONLY, device_bytes=CHUNK, dtype=E.ELLM_MXFP4)
        self.tokens = E.ellm_pool_get_geometry(probe)["tokens_per_chunk"]
        E.ellm_pool_destroy(probe)
        slots = -(-most // self.tokens)
        self.buf = torch.empty(n * slots, CHUNK, dtype=torch.uint8, device="cuda")
        self.pool = E.ellm_pool_create(self.buf, None, CHUNK, N_KV * GROUP, N_KV, DIM, n, slots, dtype=E.ELLM_MXFP4)
        self.ids = [E.ellm_tensor_create(self.pool, most) for _ in range(n)]
        self.len = np.zeros(n, np.int64)
        self.prompts = np.arange(len(prompts))
        self.forks = np.arange(len(prompts), n)

    def rows(self, n):
        return tuple(torch.randn(n, N_KV, DIM, device="cuda", generator=self.g).to(torch.bfloat16) for _ in range(2))

    def handles(self, which):
        return np.array([self.ids[i] for i in which], np.int32)

    def room(self, which, n_new):
        """Chunks for n_new more tokens of each."""
        for i, n in zip(which, n_new):
            table, _ = E.ellm_tensor_get_table(self.pool, self.ids[i])
            need = -(-int(self.len[i] + n) // self.tokens)
            have = int((table >= 0).sum())
            if need > have:
                E.ellm_tensor_map_chunks(self.pool, self.ids[i], have, need - have)

    def prompt(self, lens):
        self.room(self.prompts, lens)
        k, v = self.rows(sum(lens))
        E.ellm_kv_append(self.pool, self.handles(self.prompts), k, v, lens)
        self.len[self.prompts] = lens
        held = torch.empty_like(k), torch.empty_like(v)
        E.ellm_kv_read(self.pool, self.handles(self.prompts), *held)
        return (k, v), held

    def fork(self):
        src = np.repeat(self.prompts, self.samples)
        self.room(self.forks, self.len[src])
        E.ellm_kv_copy(self.pool, self.handles(src), self.handles(self.forks))
        self.len[self.forks] = self.len[src]

    def step(self, drafts=4):
        """Drafts, of which some are accepted, and one more token; returns the attention's queries and results."""
        ids, n = self.handles(self.forks), len(self.forks)
        self.room(self.forks, [drafts + 1] * n)
        E.ellm_kv_append(self.pool, ids, *self.rows(n * drafts), [drafts] * n)
        before = self.len[self.forks].copy()
        accepted = self.rng.integers(0, drafts + 1, n)
        # a draft may come from any branch of a tree of drafts, so the accepted ones need not be the first ones
        keep = [b + np.sort(self.rng.permutation(drafts)[:a]) for b, a in zip(before, accepted)]
        E.ellm_kv_compact(self.pool, ids, first=before, keep=torch.from_numpy(np.concatenate(keep).astype(np.int32)).cuda(), n_keep=accepted)
        self.len[self.forks] += accepted + 1
        q = torch.randn(n, N_KV * GROUP, DIM, device="cuda", generator=self.g).to(torch.bfloat16)
        out = torch.empty_like(q)
        k, v = self.rows(n)
        E.ellm_kv_append_decode(self.pool, ids, k, v, q, out)
        return q, out

    def evict(self):
        """Requests over the budget keep their first tokens and the newest half of the budget; returns how many chunks came free."""
        over = [i for i in self.forks if self.len[i] > self.budget]
        if not over:
            return 0
        n = self.budget // 2
        keep = np.concatenate([np.arange(self.len[i] - n, self.len[i]) for i in over]).astype(np.int32)
        owned = self.free()
        E.ellm_kv_compact(self.pool, self.handles(over), first=[FIRST] * len(over), keep=torch.from_numpy(keep).cuda(), n_keep=[n] * len(over),
                          flags=E.ELLM_COMPACT_UNMAP)
        self.len[over] = FIRST + n
        return self.free() - owned

    def free(self):
        return self.buf.shape[0] - sum(int((E.ellm_tensor_get_table(self.pool, t)[0] >= 0).sum()) for t in self.ids)

    def end(self):
        E.ellm_kv_compact(self.pool, self.ids, flags=E.ELLM_COMPACT_UNMAP)
        self.len[:] = 0

    def close(self):
        torch.cuda.synchronize()
        E.ellm_pool_destroy(self.pool)


def main():
    a = argparse.ArgumentParser()
    a.add_argument("--samples", type=int, default=4)
    a.add_argument("--steps", type=int, default=32)
    a = a.parse_args()
    lens = [1500, 700, 2400]
    loop = Loop(lens, a.samples, budget=2048)
    (k, _), (held, _) = loop.prompt(lens)
    error = (held.float() - k.float()).square().mean().sqrt() / k.float().square().mean().sqrt()
    print(f"prompts of {lens} tokens; {CHUNK // loop.tokens} bytes a token where bf16 takes {4 * N_KV * DIM}; rms error of the values {error:.3f}")
    loop.fork()
    for s in range(a.steps):
        _, out = loop.step()
        freed = loop.evict()
        if freed or s == a.steps - 1:
            print(f"step {s}: {int(loop.len[loop.forks].sum())} tokens of {len(loop.forks)} samples, {freed} chunks evicted, |out| {out.float().abs().mean():.4f}")
    loop.end()
    print(f"{loop.free()} of {loop.buf.shape[0]} chunks free")
    loop.close()


if __name__ == "__main__":
    main()
