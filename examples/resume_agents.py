"""Suspended agents whose KV cache is kept in fewer bits while they wait.

Each agent's context is written into a working cache (bfloat16, keys rotated on
the way).  At suspension its rows are read back and written into a retained
cache in 16, 8 or 4 bits, which is copied to host memory; at approval it is
copied back and the agent's next drafted tokens attend to it: their queries are
rotated, their keys and values written behind the context, and one
kvr_tree_attention call serves all agents, each with a tree of its own.

For every format the program prints what a token costs to keep and to restore
(the price vector of the retention controller, from the bytes of that format),
how many contexts the host tier holds, and how far the resumed attention is
from that over the unquantised cache.

    python examples/resume_agents.py [--agents 8] [--tokens 8192] [--drafts 16]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2608_30830_amd as kvr  # noqa: E402
import workloads  # noqa: E402

LAYERS, KV_HEADS, GROUP, DIM, PAGE = 32, 8, 4, 128, 64   # of the 128 KiB/token geometry


def tree_mask(drafts: int) -> list:
    """A binary tree of drafted tokens: token i follows token (i - 1) // 2."""
    seen = []
    for i in range(drafts):
        seen.append((seen[(i - 1) // 2] if i else 0) | 1 << i)
    return [m - (1 << 64) if m >> 63 else m for m in seen]


def depths(drafts: int) -> list:
    out = []
    for i in range(drafts):
        out.append(out[(i - 1) // 2] + 1 if i else 0)
    return out


class Agents:
    """Contexts of equal room in one pool, pages handed out in turn (as a server that
    serves them together would have them interleaved)."""

    def __init__(self, agents: int, tokens: int, drafts: int, seed: int):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.n, self.tokens, self.drafts = agents, tokens, drafts
        room = -(-(tokens + drafts) // PAGE)
        self.pages = agents * room
        self.page_table = (torch.arange(room, device="cuda")[None] * agents
                           + torch.arange(agents, device="cuda")[:, None]).int().contiguous()
        t = torch.arange(tokens + drafts, device="cuda")
        slots = self.page_table.long()[:, t // PAGE] * PAGE + t % PAGE
        self.slots = slots[:, :tokens].reshape(-1).contiguous()
        self.draft_slots = slots[:, tokens:].reshape(-1).contiguous()
        self.positions = t[:tokens].repeat(agents).int()
        self.draft_positions = (tokens + torch.tensor(depths(drafts), device="cuda")).repeat(agents).int()
        rows = lambda n, h: torch.randn((n, h, DIM), generator=gen, device="cuda").bfloat16()  # noqa: E731
        self.k, self.v = rows(agents * tokens, KV_HEADS), rows(agents * tokens, KV_HEADS)
        self.draft_k, self.draft_v = rows(agents * drafts, KV_HEADS), rows(agents * drafts, KV_HEADS)
        self.q = rows(agents * drafts, KV_HEADS * GROUP)
        self.cu_q = (torch.arange(agents + 1, device="cuda") * drafts).int()
        self.kv_len = torch.full((agents,), tokens + drafts, dtype=torch.int32, device="cuda")
        self.mask = torch.tensor(tree_mask(drafts), dtype=torch.int64, device="cuda").repeat(agents)[:, None]
        # positions beyond the trained 8,192 tokens by frequency blending
        self.table = kvr.kvr_rotary_table(DIM, tokens + drafts, 500000.0, kvr.KVR_ROPE_TURNS, factor=8.0,
                                          low=1.0, high=4.0, trained_len=8192.0)

    def step(self, cache: "kvr.KvCache"):
        """The drafted tokens of all agents: rotate, write, attend."""
        q = kvr.kvr_rotary(self.q, self.draft_positions, self.table, check=False)
        kvr.kvr_cache_write(cache, self.draft_k, self.draft_v, self.draft_slots, self.draft_positions,
                            self.table, check=False)
        return kvr.kvr_tree_attention(cache, q, self.cu_q, self.kv_len, self.page_table, self.drafts,
                                      self.tokens + self.drafts, tree_mask=self.mask, want_lse=True)


def main(agents: int = 8, tokens: int = 8192, drafts: int = 16, seed: int = 0, log=print) -> dict:
    if not 1 <= drafts <= 64:
        raise ValueError("1 to 64 drafted tokens")
    a = Agents(agents, tokens, drafts, seed)
    working = kvr.KvCache.allocate(kvr.KVR_KV_BF16, a.pages, KV_HEADS, PAGE, DIM)
    kvr.kvr_cache_write(working, a.k, a.v, a.slots, a.positions, a.table)
    want, want_lse = a.step(working)
    pf = workloads.PLATFORM
    found = {}
    for name, fmt in (("bf16", kvr.KVR_KV_BF16), ("fp8", kvr.KVR_KV_FP8), ("fp4", kvr.KVR_KV_FP4)):
        # suspension: the context's rows into the retained cache, and that to the host
        retained = kvr.KvCache.allocate(fmt, a.pages, KV_HEADS, PAGE, DIM)
        k, v = kvr.kvr_cache_read(working, a.slots, torch.bfloat16)
        kvr.kvr_cache_write(retained, k, v, a.slots)
        live = [t for t in retained.tensors if t is not None]
        host = [torch.empty(t.shape, dtype=t.dtype, pin_memory=True) for t in live]
        for h, t in zip(host, live):
            h.copy_(t)
        for t in live:
            t.zero_()
        # approval: back, and on with the drafted tokens
        for h, t in zip(host, live):
            t.copy_(h)
        out, lse = a.step(retained)
        per_token = kvr.kv_bytes_per_token(fmt, LAYERS, KV_HEADS, DIM)
        prices = kvr.kvr_prices_from_platform(per_token, pf["hbm_usable_bytes"], pf["host_link_bytes_per_s"],
                                              pf["prefill_tokens_per_s"], pf["n_gpu"])
        slots = int(pf["hbm_usable_bytes"] // (per_token * tokens))   # a host tier of HBM's size
        err = float((out.double() - want.double()).norm() / want.double().norm())
        found[name] = dict(bytes_per_token=per_token, b2_per_token=prices.b2_per_token, contexts=slots,
                           error=err, lse_error=float((lse - want_lse).abs().max()))
        log(f"{name}: {per_token / 1024:.0f} KiB/token, restore {tokens * prices.b2_per_token * 1e3:.1f} ms "
            f"per context, {slots} contexts in {pf['hbm_usable_bytes'] / 1e9:.0f} GB, "
            f"attention off by {err:.2e}")
    return found


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--agents", type=int, default=8)
    p.add_argument("--tokens", type=int, default=8192)
    p.add_argument("--drafts", type=int, default=16)
    main(**vars(p.parse_args()))
