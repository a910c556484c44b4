"""Several questions about one audio-visual clip, answered from an 8-bit cache of what pruning left of it.

One attention layer as an LLM's decoder runs it, on random weights: the clip's tokens are pruned by the attention its last rows pay (fastav_prune), the
survivors' K and V go into an 8-bit cache (fastav_cache_write), every question's tokens are written behind them into pages of its own and attend to
clip and question at once (fastav_attend with the clip as shared prefix), then the answers are written token by token.  In the end
the same attention is computed plainly from what fastav_cache_read gives back.

    python examples/clip_questions.py [--tokens 2048] [--keep 0.4] [--questions 8] [--answer 16] [--fp8]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_13143_b200 import fastav  # noqa: E402
from paper_2601_13143_b200.workloads import QWEN2_7B, keep_count  # noqa: E402

PAGE = 64


def _cu(counts):
    return torch.tensor([0] + list(counts), dtype=torch.int64).cumsum(0).to(torch.int32).cuda()


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def run(tokens=2048, keep=0.4, questions=8, answer=16, fp8=False, seed=0, model=QWEN2_7B):
    """The whole path; (last output, the same computed plainly, kept tokens)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, dim = model.num_q_heads, model.num_kv_heads, model.head_dim
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    # the clip: scored by its last row, pruned; K and V of the survivors go straight into the cache, by the keep list
    kept = keep_count(tokens, keep)
    q, k, v = normal(1, hq, dim), normal(tokens, hkv, dim), normal(tokens, hkv, dim)
    buf = fastav.make_buffers(q=q, q_idx=_int([tokens - 1]), cu_qlens=_cu([1]), k=k, v=None, cu_seqlens=_cu([tokens]), keep_counts=_int([kept]), lens=[tokens],
                              rows=[1], keeps=[kept])
    buf.score()
    buf.select()
    lengths = [int(n) for n in torch.randint(5, 40, (questions,), generator=gen, device="cuda")]
    clip_pages, own_pages = -(-kept // PAGE), -(-(max(lengths) + answer) // PAGE)
    cache = fastav.make_cache(clip_pages + questions * own_pages, hkv, dim, PAGE, fastav.FASTAV_CACHE_FP8 if fp8 else fastav.FASTAV_CACHE_INT8)
    clip_table = torch.arange(clip_pages, dtype=torch.int32, device="cuda")[None]
    table = torch.arange(questions * own_pages, dtype=torch.int32, device="cuda").view(questions, own_pages) + clip_pages
    clip_params = fastav.make_params(batch=1, total_tokens=tokens, max_seqlen=tokens, total_q=0, max_qlen=0, total_keep=kept, max_keep=kept, num_q_heads=hq,
                                     num_kv_heads=hkv, head_dim=dim, hidden=0, k=k, v=v)
    fastav.fastav_cache_write(clip_params, cache, k, v, buf.cu_seqlens, buf.keep_idx, buf.cu_keep, clip_table, None, status)

    prefix = dict(cu_prefix=_int([0, questions]), prefix_table=clip_table, prefix_lens=_int([kept]))
    have = [0] * questions

    def step(rows):
        """`rows` new tokens per question: into the cache behind what it has, then attention of their rows."""
        q, k, v = normal(sum(rows), hq, dim), normal(sum(rows), hkv, dim), normal(sum(rows), hkv, dim)
        params = fastav.make_params(batch=questions, total_tokens=sum(rows), max_seqlen=max(rows), total_q=0, max_qlen=0, total_keep=0, max_keep=0,
                                    num_q_heads=hq, num_kv_heads=hkv, head_dim=dim, hidden=0, k=k, v=v)
        fastav.fastav_cache_write(params, cache, k, v, _cu(rows), None, None, table, _int(have), status)
        for i, n in enumerate(rows):
            have[i] += n
        out, lse = torch.empty_like(q), torch.empty(sum(rows), hq, device="cuda")
        attend = fastav.make_attend_params(batch=questions, total_q=sum(rows), max_qlen=max(rows), num_q_heads=hq, max_kv_len=max(have), q=q, out=out,
                                           page_table=table, prefix_table=clip_table, max_prefix_len=kept, max_prefix_q=sum(rows), flags=fastav.FASTAV_CAUSAL)
        ws = torch.empty(fastav.fastav_attend_workspace_bytes(attend, cache), dtype=torch.uint8, device="cuda")
        fastav.fastav_attend(attend, cache, q, _cu(rows), table, _int(have), out, ws, lse_out_opt=lse, device_status=status, **prefix)
        return q, out

    step(lengths)                     # the questions, all their tokens at once
    for _ in range(answer):           # the answers
        q, out = step([1] * questions)

    # the last step plainly, from the rows that the cache gives back
    def read(page_table, lens):
        k, v = torch.empty(sum(lens), hkv, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(sum(lens), hkv, dim, dtype=torch.bfloat16, device="cuda")
        params = fastav.make_params(batch=len(lens), total_tokens=sum(lens), max_seqlen=max(lens), total_q=0, max_qlen=0, total_keep=0, max_keep=0,
                                    num_q_heads=hq, num_kv_heads=hkv, head_dim=dim, hidden=0, k_out=k, v_out=v)
        fastav.fastav_cache_read(params, cache, page_table, None, _cu(lens), k, v, status)
        return k.float(), v.float()

    clip_k, clip_v = read(clip_table, [kept])
    own_k, own_v = read(table, have)
    plain, at = torch.empty_like(out, dtype=torch.float32), 0
    for b, n in enumerate(have):
        k, v = torch.cat([clip_k, own_k[at:at + n]]), torch.cat([clip_v, own_v[at:at + n]])
        at += n
        for h in range(hq):
            p = torch.softmax(k[:, h // (hq // hkv)] @ q[b, h].float() / math.sqrt(dim), 0)
            plain[b, h] = p @ v[:, h // (hq // hkv)]
    if int(status):
        raise RuntimeError(f"device status {int(status)}")
    return out.float(), plain, kept


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--keep", type=float, default=0.4)
    ap.add_argument("--questions", type=int, default=8)
    ap.add_argument("--answer", type=int, default=16)
    ap.add_argument("--fp8", action="store_true")
    a = ap.parse_args()
    out, plain, kept = run(a.tokens, a.keep, a.questions, a.answer, a.fp8)
    print(f"{kept} of {a.tokens} tokens kept, {a.questions} questions, {a.answer} tokens each: "
          f"largest difference from plain attention over the cache's values {float((out - plain).abs().max()):.2e} (outputs up to {float(plain.abs().max()):.2e})")


if __name__ == "__main__":
    main()
