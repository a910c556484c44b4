"""Answers about audio-visual prompts that are written into a cache of bounded size.

One attention layer as an LLM's decoder runs it, on random weights: a prompt's queries and keys are normed per head and rotated by their positions on three axes
(fastav_rotate), the prompt is pruned by the attention its last row pays, and the survivors' K and V go into an 8-bit cache.  Then the answers are written:
every new token's rows are normed, rotated and quantised straight into the cache (fastav_rotate_write), attend to it (fastav_attend), and what they pay to
each cached token is summed up (fastav_cache_weigh); as soon as a sequence's cache is full, its lightest tokens are evicted in place, each KV head's own
(fastav_cache_evict).  In the end the same attention is computed plainly from what fastav_cache_read gives back.

    python examples/bounded_answers.py [--tokens 1500] [--keep 0.4] [--sequences 4] [--answer 64] [--budget 500] [--fp8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_13143_b200 import fastav  # noqa: E402
from paper_2601_13143_b200.workloads import QWEN2_7B, keep_count  # noqa: E402

PAGE = 32
FIRST, RECENT = 4, 32  # tokens that always stay
GRID = 12              # a frame is GRID x GRID tokens


def _cu(counts):
    return torch.tensor([0] + list(counts), dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def clip_positions(n):
    """Time, height and width of n tokens, frames of a grid behind one another: [3, n]."""
    i = torch.arange(n, device="cuda")
    return torch.stack([i // (GRID * GRID), i // GRID % GRID, i % GRID]).to(torch.int32)


def run(tokens=1500, keep=0.4, sequences=4, answer=64, budget=500, fp8=False, seed=0, model=QWEN2_7B):
    """The whole path.  Returns the last outputs, the same computed plainly, and for checks: the layer's weights and inputs, the cache read back, and which token
    (of prompt and answer, counted from 0) each KV head has in each place."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, dim = model.num_q_heads, model.num_kv_heads, model.head_dim
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    frequencies = fastav.rotary_frequencies(dim, 1e6)
    axis = [min(2, 3 * i // len(frequencies)) for i in range(len(frequencies))]
    q_norm, k_norm = 1 + normal(dim) / 8, 1 + normal(dim) / 8
    budget = max(budget, keep_count(tokens, keep) + 1)

    # the prompts: queries (of the last rows, which score) and keys in their positions, pruned, survivors into the cache
    lens, kept = [tokens] * sequences, keep_count(tokens, keep)
    k_plain, v_plain = normal(sequences * tokens, hkv, dim), normal(sequences * tokens, hkv, dim)
    pos = clip_positions(tokens)
    k, q = torch.empty_like(k_plain), normal(sequences, hq, dim)
    all_pos = pos.repeat(1, sequences)
    rotation = dict(frequencies=frequencies, axis=axis)
    fastav.fastav_rotate(fastav.make_rotate_params(k=k_plain, k_out=k, pos=all_pos, **rotation), None, k_plain, all_pos, None, k, None, k_norm)
    last_pos = pos[:, -1:].repeat(1, sequences).contiguous()
    fastav.fastav_rotate(fastav.make_rotate_params(q=q, q_out=q, pos=last_pos, **rotation), q, None, last_pos, q, None, q_norm)
    buf = fastav.make_buffers(q=q, q_idx=_int([tokens - 1] * sequences), cu_qlens=_cu([1] * sequences), k=k, v=None, cu_seqlens=_cu(lens),
                              keep_counts=_int([kept] * sequences), lens=lens, rows=[1] * sequences, keeps=[kept] * sequences)
    buf.score()
    buf.select()
    own_pages = -(-budget // PAGE)
    cache = fastav.make_cache(sequences * own_pages, hkv, dim, PAGE, fastav.FASTAV_CACHE_FP8 if fp8 else fastav.FASTAV_CACHE_INT8)
    weights = torch.zeros_like(cache.k_scale)
    table = torch.randperm(sequences * own_pages, generator=gen, device="cuda").to(torch.int32).view(sequences, own_pages)
    write = fastav.make_params(batch=sequences, total_tokens=sequences * tokens, max_seqlen=tokens, total_q=0, max_qlen=0, total_keep=sequences * kept,
                               max_keep=kept, num_q_heads=hq, num_kv_heads=hkv, head_dim=dim, hidden=0, k=k, v=v_plain)
    fastav.fastav_cache_write(write, cache, k, v_plain, buf.cu_seqlens, buf.keep_idx, buf.cu_keep, table, None, status)
    holds = buf.keep_idx.view(sequences, 1, kept).repeat(1, hkv, 1).long()  # which token lies where, per KV head

    # the answers; lengths are the same for all sequences here, and known on the host
    have, new_k, new_v = kept, [], []
    leave = max(kept, budget - budget // 8)  # an eviction makes room for some tokens at once
    rows, ones = _cu([1] * sequences), _cu([1] * sequences)
    lens_out = torch.empty(sequences, dtype=torch.int32, device="cuda")
    for step in range(answer):
        q, k, v = normal(sequences, hq, dim), normal(sequences, hkv, dim), normal(sequences, hkv, dim)
        at = torch.full((3, sequences), int(pos[0, -1]) + 1 + step, dtype=torch.int32, device="cuda")  # text: the same on all axes
        start, length = _int([have] * sequences), _int([have + 1] * sequences)
        params = fastav.make_rotate_params(q=q, k=k, v=v, q_out=q, pos=at, batch=sequences, **rotation)
        fastav.fastav_rotate_write(params, cache, q, k, v, at, ones, table, start, q, q_norm, k_norm, status)
        new_k.append(k)
        new_v.append(v)
        holds = torch.cat([holds, torch.full((sequences, hkv, 1), tokens + step, dtype=torch.int64, device="cuda")], 2)
        have += 1
        out, lse = torch.empty_like(q), torch.empty(sequences, hq, device="cuda")
        attend = fastav.make_attend_params(batch=sequences, total_q=sequences, max_qlen=1, num_q_heads=hq, max_kv_len=have, q=q, out=out, page_table=table,
                                           flags=fastav.FASTAV_CAUSAL)
        ws = torch.empty(fastav.fastav_attend_workspace_bytes(attend, cache), dtype=torch.uint8, device="cuda")
        fastav.fastav_attend(attend, cache, q, rows, table, length, out, ws, lse_out_opt=lse, device_status=status)
        fastav.fastav_cache_weigh(attend, cache, weights, q, lse, rows, table, length, start, 0.95, status)  # (the new token has no weight yet)
        if have == budget and step + 1 < answer:
            evict = fastav.make_evict_params(batch=sequences, max_kv_len=have, max_keep=leave, page_table=table, first=FIRST, recent=RECENT)
            ws = torch.empty(fastav.fastav_evict_workspace_bytes(evict, cache), dtype=torch.uint8, device="cuda")
            idx = torch.empty(sequences, hkv, leave, dtype=torch.int32, device="cuda")
            fastav.fastav_cache_evict(evict, cache, weights, table, length, _int([leave] * sequences), lens_out, ws, keep_idx_out_opt=idx, device_status=status)
            holds = holds.gather(2, idx.long())
            have = leave

    # the last step plainly, from the rows that the cache gives back
    ck, cv = (torch.empty(sequences * have, hkv, dim, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    read = fastav.make_params(batch=sequences, total_tokens=sequences * have, max_seqlen=have, total_q=0, max_qlen=0, total_keep=0, max_keep=0, num_q_heads=hq,
                              num_kv_heads=hkv, head_dim=dim, hidden=0, k_out=ck, v_out=cv)
    fastav.fastav_cache_read(read, cache, table, None, _cu([have] * sequences), ck, cv, status)
    if int(status):
        raise RuntimeError(f"device status {int(status)}")
    ck, cv = ck.view(sequences, have, hkv, dim), cv.view(sequences, have, hkv, dim)
    group = hq // hkv
    z = torch.einsum("bhd,bnhd->bhn", q.float(), ck.float().repeat_interleave(group, 2)) / math.sqrt(dim)
    plain = torch.einsum("bhn,bnhd->bhd", torch.softmax(z, 2), cv.float().repeat_interleave(group, 2))
    state = dict(k_norm=k_norm, frequencies=frequencies, axis=axis, pos=pos, k=k_plain.view(sequences, tokens, hkv, dim), v=v_plain.view(sequences, tokens, hkv, dim),
                 new_k=torch.stack(new_k, 1), new_v=torch.stack(new_v, 1), cache_k=ck, cache_v=cv, holds=holds, lens=have)
    return out.float(), plain, state


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=1500)
    ap.add_argument("--keep", type=float, default=0.4)
    ap.add_argument("--sequences", type=int, default=4)
    ap.add_argument("--answer", type=int, default=64)
    ap.add_argument("--budget", type=int, default=640)
    ap.add_argument("--fp8", action="store_true")
    a = ap.parse_args()
    out, plain, state = run(a.tokens, a.keep, a.sequences, a.answer, a.budget, a.fp8)
    print(f"{a.sequences} prompts of {a.tokens} tokens, {a.answer} new tokens each, {state['lens']} cached in the end: "
          f"largest difference from plain attention over the cache's values {float((out - plain).abs().max()):.2e} (outputs up to {float(plain.abs().max()):.2e})")


if __name__ == "__main__":
    main()
