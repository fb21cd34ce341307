"""A long context through one layer: kept in a paged cache, indexed by its keys' features, and answered from a part of it.

  prefill   chunk by chunk: keys and values appended (rotated on the way), the chunk attends to everything so far; the same
            keys, before rotation, are encoded by the sparse autoencoder and indexed
  look-up   the question's queries score all positions in the index; its evidence spans name blocks of the cache
  answer    token by token: append, then attention over the spans' blocks, the first block and the newest ones (one
            list for all heads), and over the blocks that each step's own queries choose by the pages' signatures

With eight_bits the cache is one of 8 bits, keys and queries are normed for each head on the way in, scores are capped, and at the end the spans' tokens are
read back into a small cache of their own, whose attention needs nothing of the large one.

Run with `python examples/paged_answer.py` (`--eight-bits`).  Activations are random with some structure: no weights are needed.  What is printed is the
share of the full attention's weight that each kind of list holds, from the log-sum-exps of the three calls.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_17702_amd as s3  # noqa: E402


def span_blocks(starts, span_len: int, page: int, last_block: int, top: int, device):
    """The first block and the newest two, then the blocks that the spans lie in, best span first, as far as `top` goes (top >= 3): each
    once, in ascending order, -1 filled: [top] int32."""
    per = (span_len + page - 2) // page + 1
    blk = torch.div(starts, page, rounding_mode="floor")[:, None] + torch.arange(per, device=device)[None]
    out_of_span = (starts < 0)[:, None] | (blk * page >= starts[:, None] + span_len) | (blk > last_block)
    blk = torch.cat([torch.tensor([0, last_block, max(last_block - 1, 0)], device=device), blk.masked_fill(out_of_span, 0).flatten()])
    none = blk.numel()
    at = torch.full((last_block + 1,), none, device=device).scatter_reduce(0, blk, torch.arange(none, device=device), "amin")     # first named where
    at, order = at.sort()
    order = torch.where(at < none, order, last_block + 1)[:top].sort().values
    out = torch.full((top,), -1, dtype=torch.int32, device=device)
    out[:order.numel()] = torch.where(order <= last_block, order, -1).to(torch.int32)
    return out


def run(context: int = 8192, chunk: int = 2048, answer: int = 8, n_q: int = 32, n_kv: int = 8, d: int = 128, page: int = 64,
        n_feat: int = 4096, k: int = 32, top_blocks: int = 32, span: int = 64, n_spans: int = 12, seed: int = 0, device="cuda",
        eight_bits: bool = False, softcap: float = 30.0):
    g = torch.Generator(device=device).manual_seed(seed)
    bf = torch.bfloat16

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=device)

    # a few topics; the tokens of a stretch of the context, and the question, follow one each
    topics = normal(16, n_kv, d)
    topic_of = (torch.arange(context + chunk, device=device) // 256) % 16

    def project(n, topic):
        """Queries, keys and values of n tokens, side by side as one projection gives them."""
        qkv = normal(n, n_q + 2 * n_kv, d) * 0.7
        lean = topics[topic]
        qkv[:, n_q:n_q + n_kv] += lean
        qkv[:, :n_q] += lean.repeat_interleave(n_q // n_kv, dim=1)
        return qkv.to(bf)

    total = context + answer
    pages = -(-total // page)
    if eight_bits:
        cache = s3.KVCache8(pages, page, n_kv, d, signatures=True, device=device)
        norms = {"q_norm": 1.0 + 0.1 * normal(d), "k_norm": 1.0 + 0.1 * normal(d)}
        capped = {"softcap": softcap}
    else:
        cache, norms, capped = s3.KVCache(pages, page, n_kv, d, bf, signatures=True, device=device), {}, {}
    table = torch.randperm(pages, generator=g, device=device).to(torch.int32)[None]
    rope = s3.rope_table(total, d, device=device)
    w_enc = torch.nn.functional.normalize(normal(n_kv, n_feat, d), dim=-1).to(bf)
    b_enc = torch.zeros(n_kv, n_feat, device=device)
    index = s3.Index(n_kv, n_feat, k, context)
    tau = s3.new_tau_hint(n_kv, device)

    # prefill
    for c0 in range(0, context, chunk):
        n = min(chunk, context - c0)
        qkv = project(n, topic_of[c0:c0 + n])
        q, keys, v = qkv[:, :n_q], qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:]
        kv_len = torch.tensor([c0 + n], dtype=torch.int32, device=device)
        q_start = torch.tensor([0, n], dtype=torch.int32, device=device)
        q = cache.append(keys, v, kv_len, table, q_start=q_start, rope=rope, q=q, **norms)
        hidden, _ = cache.attention(q, kv_len, table, q_start=q_start, max_new=n, max_kv=c0 + n, **capped)
        ids, _ = s3.sae_encode_topk_stream(keys.transpose(0, 1).contiguous(), w_enc, b_enc, k, tau)
        index.append(ids, base_pos=c0)
    index.finalize()

    # look-up: the question is about topic 5
    asked = project(16, torch.full((16,), 5, device=device))[:, :n_q]
    per_head = asked.view(16, n_kv, n_q // n_kv, d).permute(1, 0, 2, 3).reshape(n_kv, -1, d).contiguous()
    qids, qvals = s3.sae_encode_topk(per_head, w_enc, b_enc, k)
    starts, _, _, _ = index.coactivate_score(qids, qvals, context, span, n_spans)

    # answer
    shares = {"span_share": [], "chosen_share": []}
    for t in range(answer):
        qkv = project(1, torch.full((1,), 5, device=device))
        length = context + t + 1
        kv_len = torch.tensor([length], dtype=torch.int32, device=device)
        q = cache.append(qkv[:, n_q:n_q + n_kv], qkv[:, n_q + n_kv:], kv_len, table, rope=rope, q=qkv[:, :n_q], **norms)
        full, lse = cache.attention(q, kv_len, table, max_kv=length, want_lse=True, **capped)
        last = (length - 1) // page
        named = span_blocks(starts, span, page, last, top_blocks, device).expand(1, n_kv, top_blocks).contiguous()
        _, lse_named = cache.block_attention(q, kv_len, table, named, want_lse=True, **capped)
        chosen = cache.select(q, kv_len, table, top_blocks, lead=1, tail=2, max_kv=length)
        _, lse_chosen = cache.block_attention(q, kv_len, table, chosen, want_lse=True, **capped)
        shares["span_share"].append(torch.exp(lse_named - lse).mean())
        shares["chosen_share"].append(torch.exp(lse_chosen - lse).mean())
    kept = {}
    if eight_bits:
        # the evidence alone: the spans' tokens, rotated as they are, in a cache of their own
        lo = starts.clamp(min=0)
        _, idx, n_out = s3.fuse_indices(context, lo, torch.where(starts < 0, lo - 1, torch.clamp(lo + span - 1, max=context - 1)), None, lead=1)
        n = int(n_out)
        k, v = cache.read(kv_len, table, n, q_start=torch.tensor([0, n], dtype=torch.int32, device=device), positions=idx[:n])
        small = s3.KVCache8(-(-n // page), page, n_kv, d, device=device)
        small_table = torch.arange(small.n_pages, dtype=torch.int32, device=device)[None]
        small_len = torch.tensor([n], dtype=torch.int32, device=device)
        small.append(k, v, small_len, small_table, q_start=torch.tensor([0, n], dtype=torch.int32, device=device))
        out, lse_kept = small.attention(q, small_len, small_table, max_kv=n, want_lse=True, **capped)
        kept = {"kept": out, "kept_tokens": n, "kept_k": k, "small": small, "kept_share": float(torch.exp(lse_kept - lse).mean())}
    return {**kept, "hidden": hidden, "full": full, "starts": starts, "named": named, "chosen": chosen, "blocks": last + 1,
            **{name: float(torch.stack(x).mean()) for name, x in shares.items()}}


if __name__ == "__main__":
    r = run(eight_bits="--eight-bits" in sys.argv[1:])
    print(f"{r['blocks']} blocks in the cache, lists of {r['chosen'].shape[2]}: the blocks of the evidence spans hold {r['span_share']:.2f} of the full "
          f"attention's weight, those that each step chooses {r['chosen_share']:.2f} (their part of the cache: {r['chosen'].shape[2] / r['blocks']:.2f})")
    if "kept" in r:
        print(f"{r['kept_tokens']} tokens of the spans, read back into a cache of their own, hold {r['kept_share']:.2f} of it")
