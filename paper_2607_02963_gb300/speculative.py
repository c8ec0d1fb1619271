"""Speculative steps of event branches: drafted tokens of every branch are written into the paged cache, attended
together, verified against the target's probabilities, and the branches advance by what was kept.

``BranchCache`` holds what a program keeps for one attention layer (pools in bf16 or 8 bits, page table, page
bookkeeping, lengths); a step is ``plan`` -> ``append`` -> ``attend`` -> ``verify`` -> ``commit``, each one call of the
C ABI.  A model of many layers shares one plan and page table among its layers' pools.

    python -m paper_2607_02963_gb300.speculative        (a GPU; synthetic tensors, no model)

runs such steps for a few branches over a shared prefix and prints what they keep.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


class BranchCache:
    """The private cache of a layer's event branches and the steps on it."""

    def __init__(self, h_q, h_kv, head_dim, n_events, n_pages, max_pages, page_size=16, kv_format=B.KV_FP8,
                 prefix_len=None, event_video=None, out_dtype=1, device="cuda"):
        self.problem = B.make_problem(h_q, h_kv, head_dim, page_size, out_dtype=out_dtype)
        self.kv_format, self.device = kv_format, torch.device(device)
        self.prefix_len, self.event_video = prefix_len, event_video
        shape = (n_pages, h_kv, page_size, head_dim)
        kind = torch.uint8 if kv_format == B.KV_FP8 else torch.bfloat16
        self.k_pool, self.v_pool = (torch.zeros(shape, dtype=kind, device=self.device) for _ in range(2))
        self.k_scale = self.v_scale = None
        if kv_format == B.KV_FP8:
            self.k_scale, self.v_scale = (torch.zeros(shape[:3], dtype=torch.uint8, device=self.device) for _ in range(2))
        self.page_table = torch.full((n_events, max_pages), -1, dtype=torch.int32, device=self.device)
        self.pages = B.CacheState(n_pages)
        self.event_len = np.zeros(n_events, dtype=np.int32)
        self.workspace = None

    def plan(self, n_new) -> B.ChunkPlan:
        """Plan a step of n_new[e] tokens per branch (drafted tokens after each branch's last accepted one, or a
        prompt's chunk); takes the pages they start."""
        n_new = np.ascontiguousarray(n_new, dtype=np.int32)
        need = B.pad_chunk_workspace_size(self.problem, self.prefix_len, self.event_video, self.event_len, n_new,
                                          kv_format=self.kv_format)
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = torch.zeros(need, dtype=torch.uint8, device=self.device)
        return B.pad_chunk_plan(self.problem, self.pages, self.prefix_len, self.event_video, self.event_len, n_new,
                                page_table=self.page_table, kv_format=self.kv_format, workspace=self.workspace)

    def append(self, plan, k_new, v_new):
        B.pad_chunk_append(plan, k_new, v_new, self.k_pool, self.v_pool, self.k_scale, self.v_scale)

    def attend(self, plan, q, k_prefix=None, v_prefix=None, out=None, lse=None):
        if out is None:
            kind = torch.bfloat16 if self.problem.out_dtype == 1 else torch.float32
            out = torch.empty(q.shape, dtype=kind, device=self.device)
        B.pad_chunk_attn(plan, q, k_prefix, v_prefix, self.k_pool, self.v_pool, out, lse, self.k_scale, self.v_scale)
        return out

    def read(self, plan):
        """The branches' cached tokens as contiguous bf16 (k, v), branch after branch: the layout of a prefix."""
        shape = (plan.n_cached, self.problem.h_kv, self.problem.head_dim)
        k, v = (torch.empty(shape, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        B.pad_chunk_read(plan, self.k_pool, self.v_pool, k, v, self.k_scale, self.v_scale)
        return k, v

    def verify(self, plan, p, q, draft, u_accept, u_pick):
        """(accepted, token) of every branch, on the device."""
        accepted, token = (torch.empty(plan.n_events, dtype=torch.int32, device=self.device) for _ in range(2))
        B.pad_draft_verify(plan, p, q, draft, u_accept, u_pick, accepted, token)
        return accepted, token

    def commit(self, plan, accepted=None):
        """Advance the branches by their accepted drafts and the token before them; other new pages go back."""
        if accepted is not None:
            accepted = accepted.cpu().numpy()
        self.event_len = plan.commit(self.pages, accepted)
        return self.event_len


def example(events=6, drafts=4, steps=5, prefix=2048, vocab=4096, kv_format=B.KV_FP8, h_q=28, h_kv=4, head_dim=128, seed=0):
    """A few speculative steps on synthetic tensors; returns the kept tokens per step and the final lengths."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()

    cache = BranchCache(h_q, h_kv, head_dim, events, n_pages=events * 16, max_pages=16, kv_format=kv_format,
                        prefix_len=[prefix], event_video=[0] * events)
    k_prefix, v_prefix = randn(prefix, h_kv, head_dim), randn(prefix, h_kv, head_dim)
    kept = []
    for _ in range(steps):
        plan = cache.plan([drafts + 1] * events)
        n = plan.n_tokens
        cache.append(plan, randn(n, h_kv, head_dim), randn(n, h_kv, head_dim))
        out = cache.attend(plan, randn(n, h_q, head_dim), k_prefix, v_prefix)
        # stand-ins for the target's and the draft's distributions: the same logits, one with an error
        logits = 3.0 * torch.randn(n, vocab, generator=g, device="cuda")
        p = torch.softmax(logits, -1)
        rows = torch.arange(n, device="cuda").view(events, drafts + 1)[:, :drafts].reshape(-1)
        q = torch.softmax(logits[rows] + 0.5 * torch.randn(len(rows), vocab, generator=g, device="cuda"), -1)
        draft = torch.multinomial(q, 1, generator=g)[:, 0].to(torch.int32)
        accepted, _token = cache.verify(plan, p, q, draft, torch.rand(len(rows), generator=g, device="cuda"),
                                        torch.rand(events, generator=g, device="cuda"))
        B.pad_chunk_status(plan)
        if not bool(torch.isfinite(out).all()):
            raise RuntimeError("attention returned values that are not finite")
        cache.commit(plan, accepted)
        kept.append((accepted + 1).tolist())
    return kept, cache


def main():
    for name, fmt in (("bf16", B.KV_BF16), ("8 bits", B.KV_FP8)):
        kept, cache = example(kv_format=fmt)
        print(f"cache in {name}:")
        for i, row in enumerate(kept):
            print(f"  step {i}: tokens kept per branch {row}")
        print(f"  lengths {cache.event_len.tolist()}, {cache.pages.n_pages - cache.pages.free_count} pages in use")


if __name__ == "__main__":
    main()
