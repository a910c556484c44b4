"""The work of the 8-bit K/V cache as measurable cases: survivors quantised into its pages, rows read back, and attention over it, with
and without a prefix that several sequences share.

Sizes are those of the package's workloads (``workloads.py``), or generic ones of the same kind; ``draw`` spreads over the same ranges.
Values are made on the GPU from the seed, with the heavy-tailed token importance of audio-visual prompts: keys carry a per-token
component along a direction that all query rows share, and a few early anchor tokens carry a large one.
"""
import math
import random

import torch

own = False

# (query heads, KV heads, head_dim): the three decoder shapes of the workloads, then two generic ones
TINY = (8, 2, 64)
QWEN2 = (28, 4, 128)
MISTRAL = (32, 8, 128)
SHAPES = (TINY, QWEN2, MISTRAL, (16, 16, 64), (32, 4, 128))

LOGIT_SPREAD = 1.5  # standard deviation of a token's shared logit shift
SHARED = 0.5        # share of a query that is common to all rows and heads of a KV group

LARGEST = {"int8": 127.0, "fp8": 448.0}  # a row's largest magnitude is laid on this code


def _case(name, kind, shape, **more):
    hq, hkv, dim = shape
    c = {"kind": kind, "q_heads": hq, "kv_heads": hkv, "dim": dim, **more}
    return {"name": name, **c} if name else c


def _write(name, shape, fmt, page, batch, lo, hi, layout, keep_lo=0.0, keep_hi=0.0, start_hi=0, packed=False):
    """`keep_lo` 0: every row, else a keep list. `start_hi`: most tokens that a sequence has in the cache before."""
    return _case(name, "write", shape, format=fmt, page=page, batch=batch, lo=lo, hi=hi, layout=layout, keep_lo=keep_lo, keep_hi=keep_hi,
                 start_hi=start_hi, packed=packed)


def _read(name, shape, fmt, page, batch, lo, hi, layout, start_hi=0):
    return _case(name, "read", shape, format=fmt, page=page, batch=batch, lo=lo, hi=hi, layout=layout, start_hi=start_hi)


def _attend(name, shape, fmt, page, batch, lo, hi, rows_lo, rows_hi, layout, prefixes=0, plo=0, phi=0):
    """`lo`..`hi`: a sequence's own tokens, its rows (the last of them) included; `prefixes` groups with a prefix of `plo`..`phi`."""
    return _case(name, "attend", shape, format=fmt, page=page, batch=batch, lo=lo, hi=hi, rows_lo=rows_lo, rows_hi=rows_hi, layout=layout,
                 prefixes=prefixes, plo=plo, phi=phi)


def listed():
    return [
        # a layer's survivors of four long clips (40 % kept) go into its cache
        _write("write_survivors_4x16384", MISTRAL, "int8", 64, 4, 16384, 16384, 0, keep_lo=0.4, keep_hi=0.4),
        # ... and those of a ragged serving batch, K and V as views of a packed projection
        _write("write_survivors_ragged_32", QWEN2, "fp8", 128, 32, 1024, 8192, 1, keep_lo=0.3, keep_hi=0.7, packed=True),
        # one decoding step's token of 32 sequences, behind what they have (latency)
        _write("write_token_32", QWEN2, "fp8", 16, 32, 1, 1, 2, start_hi=4096, packed=True),
        # one prompt's rows back in bf16, for a later prune call
        _read("read_1x2230", QWEN2, "fp8", 64, 1, 2230, 2230, 3),
        # a batch's, from the middle of their pages on
        _read("read_ragged_32", QWEN2, "int8", 64, 32, 512, 4096, 4, start_hi=100),
        # the smallest attention: one sequence's next token over a thousand survivors (latency)
        _attend("answer_1x1024", QWEN2, "int8", 64, 1, 1024, 1024, 1, 1, 5),
        # the next token of 32 ragged sequences
        _attend("answer_ragged_32", QWEN2, "fp8", 64, 32, 512, 4096, 1, 1, 6),
        # the next token of four clips that were not pruned
        _attend("answer_4x16384", MISTRAL, "int8", 256, 4, 16384, 16384, 1, 1, 7),
        # a few drafted tokens each of eight sequences of a small decoder, causal among themselves
        _attend("drafts_8x744", TINY, "fp8", 16, 8, 500, 744, 2, 8, 8),
        # 32 answers being written about one long clip, which all of them read
        _attend("shared_answer_32_on_16384", MISTRAL, "int8", 64, 32, 16, 256, 1, 1, 9, prefixes=1, plo=16384, phi=16384),
        # 24 sequences on three pruned clips, a few drafted tokens each
        _attend("shared_drafts_24_on_3", QWEN2, "fp8", 32, 24, 20, 300, 1, 8, 10, prefixes=3, plo=2048, phi=6554),
        # the questions themselves: all tokens of 16 questions about one long clip at once (the largest)
        _attend("shared_questions_16_on_16384", MISTRAL, "int8", 64, 16, 64, 128, 64, 128, 11, prefixes=1, plo=16384, phi=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("write", "write", "read", "attend", "attend", "attend", "shared", "shared", "shared"))
    shape, fmt, page, layout = rng.choice(SHAPES), rng.choice(("int8", "fp8")), rng.choice((16, 32, 64, 128, 256)), rng.randrange(1 << 20)
    if kind in ("write", "read"):
        total = _log_int(rng, 16, 60000)  # rows of the batch
        batch = min(_log_int(rng, 1, 64), total)
        hi = max(1, total // batch)
        lo = max(1, int(hi * rng.uniform(0.2, 1.0)))
        start = rng.choice((0, _log_int(rng, 1, 2000)))
        if kind == "read":
            return _read("", shape, fmt, page, batch, lo, hi, layout, start_hi=start)
        keep = rng.choice((0.0, round(rng.uniform(0.2, 0.8), 3)))
        return _write("", shape, fmt, page, batch, lo, hi, layout, keep_lo=keep, keep_hi=min(0.9, keep + 0.2) if keep else 0.0, start_hi=start,
                      packed=rng.random() < 0.5)
    batch = _log_int(rng, 1, 64)
    rows_hi = rng.choice((1, 1, _log_int(rng, 2, 8), _log_int(rng, 9, 128)))
    rows_lo = max(1, int(rows_hi * rng.uniform(0.2, 1.0)))
    prefixes = plo = phi = 0
    if kind == "shared":
        prefixes = min(batch, rng.choice((1, 1, 1, rng.randint(2, 4))))
        phi = _log_int(rng, 200, 16384)
        plo = max(1, int(phi * rng.uniform(0.4, 1.0)))
        lo, hi = rows_lo, rows_hi + _log_int(rng, 1, 400)
    else:
        hi = max(rows_hi, _log_int(rng, 100, 16384))
        lo = max(rows_lo, int(hi * rng.uniform(0.2, 1.0)))
        batch = min(batch, max(1, 131072 // hi))
    # no more than the largest listed case has in logits, nor in keys of the plain form
    batch = max(1, min(batch, (1 << 29) // (rows_hi * shape[0] * (hi + phi))))
    prefixes = min(prefixes, batch)
    return _attend("", shape, fmt, page, batch, lo, hi, rows_lo, rows_hi, layout, prefixes=prefixes, plo=plo, phi=phi)


# ---- sizes (a case fixes them; only the values come from the seed) -----------------------------------

def _sizes(case):
    rng = random.Random(case["layout"])
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    s = {"lens": n, "start": [rng.randint(0, case["start_hi"]) for _ in n] if case.get("start_hi") else [0] * len(n)}
    s["count"] = [max(1, int(m * rng.uniform(case["keep_lo"], case["keep_hi"]))) for m in n] if case.get("keep_lo") else list(n)
    if case["kind"] == "attend":
        s["rows"] = [min(m, rng.randint(case["rows_lo"], case["rows_hi"])) for m in n]
        groups = case["prefixes"]
        s["prefix_lens"] = [rng.randint(case["plo"], case["phi"]) for _ in range(groups)]
        s["cu_prefix"] = [round(i * len(n) / groups) for i in range(groups + 1)] if groups else [0]
    return s


def _cu(counts):
    cu = [0]
    for c in counts:
        cu.append(cu[-1] + c)
    return cu


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- values -------------------------------------------------------------------------------------------

def _keys(gen, case, tokens, shared, anchors=16):
    hkv, dim = case["kv_heads"], case["dim"]
    shift = torch.randn(tokens, generator=gen, device="cuda")
    early = torch.randperm(max(1, tokens // 4), generator=gen, device="cuda")[:min(anchors, tokens // 16)]
    shift[early] = 3.0
    k = torch.randn(tokens, hkv, dim, generator=gen, device="cuda")
    return k + (shift * (LOGIT_SPREAD / (SHARED * math.sqrt(dim))))[:, None, None] * shared


def _codes(case, x):
    """A cache's content for rows x [..., dim]: codes and scales, as an earlier write left them."""
    top = x.abs().amax(-1)
    y = x * (LARGEST[case["format"]] / top)[..., None]
    return (y.round().to(torch.int8) if case["format"] == "int8" else y.to(torch.float8_e4m3fn)), top / LARGEST[case["format"]]


def _tables(gen, case, tokens, used=0):
    """Page table [rows, most pages] for sequences of that many tokens, pages in no order; -1 where a sequence has none."""
    need = [-(-n // case["page"]) for n in tokens]
    ids = used + torch.randperm(sum(need), generator=gen, device="cuda")
    table = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    cu = _cu(need)
    for b, m in enumerate(need):
        table[b, :m] = ids[cu[b]:cu[b + 1]]
    return table, used + sum(need)


def _pool(case, pages, parts):
    """Pools [pages, KV heads, page tokens, dim] and scales without the last, filled from (table, lengths, rows of all sequences)."""
    hkv, dim, page = case["kv_heads"], case["dim"], case["page"]
    code = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    pools = [torch.zeros(pages, hkv, page, dim, dtype=torch.int8, device="cuda").view(code) for _ in "kv"]
    scales = [torch.zeros(pages, hkv, page, device="cuda") for _ in "kv"]
    for table, lens, both in parts:
        b = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).cuda()
        at = torch.cat([torch.arange(n) for n in lens]).cuda()
        to = table[b, at // page].long()
        for pool, scale, x in zip(pools, scales, both):
            c, s = _codes(case, x)
            pool.view(torch.int8)[to, :, at % page] = c.view(torch.int8)
            scale[to, :, at % page] = s
    return {"k_pool": pools[0], "v_pool": pools[1], "k_scale": scales[0], "v_scale": scales[1]}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    s = _sizes(case)
    state = {"kind": case["kind"], "format": case["format"], "hkv": hkv, "hq": hq, "dim": dim, "page": case["page"], "sizes": s}
    shared = torch.randn(hkv, dim, generator=gen, device="cuda")
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    if case["kind"] == "write":
        total = sum(s["lens"])
        k = torch.cat([_keys(gen, case, n, shared) for n in s["lens"]]).to(torch.bfloat16)
        v = normal(total, hkv, dim).to(torch.bfloat16)
        if case["packed"]:
            whole = torch.zeros(total, hq + 2 * hkv, dim, dtype=torch.bfloat16, device="cuda")
            whole[:, hq:hq + hkv], whole[:, hq + hkv:] = k, v
            k, v = whole[:, hq:hq + hkv], whole[:, hq + hkv:]
        if case["keep_lo"]:
            state["keep_idx"] = torch.cat([torch.randperm(n, generator=gen, device="cuda")[:c].sort().values for n, c in zip(s["lens"], s["count"])]).to(torch.int32)
            state["cu_keep"] = _int(_cu(s["count"]))
        table, pages = _tables(gen, case, [a + c for a, c in zip(s["start"], s["count"])])
        state.update(k=k, v=v, cu_seqlens=_int(_cu(s["lens"])), start=_int(s["start"]), table=table, **_pool(case, pages, []))
    elif case["kind"] == "read":
        lens = [a + c for a, c in zip(s["start"], s["lens"])]
        table, pages = _tables(gen, case, lens)
        rows = (torch.cat([_keys(gen, case, n, shared) for n in lens]), normal(sum(lens), hkv, dim))
        new = lambda: torch.empty(sum(s["lens"]), hkv, dim, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        state.update(cu_seqlens=_int(_cu(s["lens"])), start=_int(s["start"]), table=table, k_out=new(), v_out=new(), **_pool(case, pages, [(table, lens, rows)]))
    else:
        rows, lens, plens = s["rows"], s["lens"], s["prefix_lens"]
        table, pages = _tables(gen, case, lens)
        parts = [(table, lens, (torch.cat([_keys(gen, case, n, shared) for n in lens]), normal(sum(lens), hkv, dim)))]
        if plens:
            ptable, pages = _tables(gen, case, plens, pages)
            parts.append((ptable, plens, (torch.cat([_keys(gen, case, n, shared) for n in plens]), normal(sum(plens), hkv, dim))))
            state.update(prefix_table=ptable, prefix_lens=_int(plens), cu_prefix=_int(s["cu_prefix"]))
        q = normal(sum(rows), hkv, hq // hkv, dim) * math.sqrt(1 - SHARED ** 2) + SHARED * shared[:, None, :]
        state.update(q=q.reshape(sum(rows), hq, dim).to(torch.bfloat16), cu_qlens=_int(_cu(rows)), table=table, kv_lens=_int(lens),
                     out=torch.empty(sum(rows), hq, dim, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(sum(rows), hq, device="cuda"),
                     **_pool(case, pages, parts))
    return state


# ---- the framework's operators -------------------------------------------------------------------------

def _handle(state):
    """What a program makes once: the cache's handle, parameters, workspace."""
    if "cache" not in state:
        from paper_2601_13143_b200 import fastav as F
        s = state["sizes"]
        state["F"] = F
        state["cache"] = F.KvCache(state["k_pool"], state["v_pool"], state["k_scale"], state["v_scale"])
        if state["kind"] == "attend":
            groups, n = s["cu_prefix"], s["rows"]
            state["params"] = F.make_attend_params(
                batch=len(n), total_q=sum(n), max_qlen=max(n), num_q_heads=state["hq"], max_kv_len=max(s["lens"]), q=state["q"], out=state["out"],
                page_table=state["table"], prefix_table=state.get("prefix_table"), max_prefix_len=max(s["prefix_lens"], default=0),
                max_prefix_q=max((sum(n[a:b]) for a, b in zip(groups, groups[1:])), default=0), flags=F.FASTAV_CAUSAL)
            state["workspace"] = torch.empty(F.fastav_attend_workspace_bytes(state["params"], state["cache"]), dtype=torch.uint8, device="cuda")
        else:
            counts, listed_rows = s["count"], "keep_idx" in state
            state["params"] = F.make_params(
                batch=len(counts), total_tokens=sum(s["lens"]), max_seqlen=max(s["lens"]), total_q=0, max_qlen=0,
                total_keep=sum(counts) if listed_rows else 0, max_keep=max(counts) if listed_rows else 0, num_q_heads=state["hq"],
                num_kv_heads=state["hkv"], head_dim=state["dim"], hidden=0, k=state.get("k"), v=state.get("v"), k_out=state.get("k_out"),
                v_out=state.get("v_out"))
    return state["F"], state["cache"], state["params"]


def _run_own(s):
    F, cache, params = _handle(s)
    if s["kind"] == "write":
        F.fastav_cache_write(params, cache, s["k"], s["v"], s["cu_seqlens"], s.get("keep_idx"), s.get("cu_keep"), s["table"], s["start"])
        return _pools(s)
    if s["kind"] == "read":
        F.fastav_cache_read(params, cache, s["table"], s["start"], s["cu_seqlens"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    F.fastav_attend(params, cache, s["q"], s["cu_qlens"], s["table"], s["kv_lens"], s["out"], s["workspace"], cu_prefix=s.get("cu_prefix"),
                    prefix_table=s.get("prefix_table"), prefix_lens=s.get("prefix_lens"), lse_out_opt=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


# ---- their plain forms -----------------------------------------------------------------------------------

def _pools(s):
    """The whole cache: int8 codes are whole numbers, e4m3 codes the values of their type, both in units of the scales."""
    return {"k": s["k_pool"], "v": s["v_pool"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _spread(cu, total):
    """Of packed rows: the sequence, and the place in it."""
    counts = (cu[1:] - cu[:-1]).long()
    b = torch.repeat_interleave(torch.arange(len(counts), device=cu.device), counts, output_size=total)
    return b, torch.arange(total, device=cu.device) - cu.long()[b]


def _plain_write(s):
    cu = s["cu_keep"] if "keep_idx" in s else s["cu_seqlens"]
    b, i = _spread(cu, sum(s["sizes"]["count"]))
    src = s["cu_seqlens"].long()[b] + (s["keep_idx"].long() if "keep_idx" in s else i)
    at = s["start"].long()[b] + i
    page, slot = s["table"][b, at // s["page"]].long(), at % s["page"]
    largest = LARGEST[s["format"]]
    for name in "kv":
        x = s[name][src].float()
        top = x.abs().amax(-1)
        y = torch.where(top[..., None] == 0, torch.zeros_like(x), x * largest / top[..., None])
        code = y.round().clamp(-127, 127).to(torch.int8) if s["format"] == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.int8)
        s[name + "_pool"].view(torch.int8)[page, :, slot] = code
        s[name + "_scale"][page, :, slot] = top / largest
    return _pools(s)


def _plain_read(s):
    b, i = _spread(s["cu_seqlens"], sum(s["sizes"]["lens"]))
    at = s["start"].long()[b] + i
    page, slot = s["table"][b, at // s["page"]].long(), at % s["page"]
    for name in "kv":
        code = s[name + "_pool"].view(torch.int8)[page, :, slot].view(s[name + "_pool"].dtype)
        s[name + "_out"].copy_(code.float() * s[name + "_scale"][page, :, slot][..., None])
    return {"k": s["k_out"], "v": s["v_out"]}


def _dense(s, name, table):
    """[rows of the table, KV heads, tokens, dim] in fp32, padded to the longest."""
    at = table.clamp(min=0).long()
    pool = s[name + "_pool"]
    x = pool.view(torch.int8)[at].view(pool.dtype).float() * s[name + "_scale"][at][..., None]   # [rows, pages, heads, tokens, dim]
    return x.transpose(1, 2).reshape(len(table), s["hkv"], -1, s["dim"])


def _padded(s, at, there):
    """Query rows gathered to [groups, KV heads, rows x G, dim], zero where there is none."""
    q = s["q"].float()[at] * there[..., None, None]
    return q.view(*at.shape, s["hkv"], -1, s["dim"]).permute(0, 2, 1, 3, 4).flatten(2, 3)


def _plain_attend(s):
    total, hq, hkv, dim = len(s["q"]), s["hq"], s["hkv"], s["dim"]
    sizes, cu = s["sizes"], s["cu_qlens"].long()
    parts = []  # (table, lengths, index of the padded rows, which of them are there, most keys each of them sees)

    def part(table, lens, first, count, most_rows, causal):
        i = torch.arange(most_rows, device="cuda")
        there = i < count[:, None]
        sees = (lens[:, None] - count[:, None] + i + 1).clamp(min=0) if causal else lens[:, None].expand(-1, most_rows)
        parts.append((table, (first[:, None] + i).clamp(max=total - 1), there, sees))

    part(s["table"], s["kv_lens"].long(), cu[:-1], cu[1:] - cu[:-1], max(sizes["rows"]), True)
    if "cu_prefix" in s:
        edges = cu[s["cu_prefix"].long()]
        groups = sizes["cu_prefix"]
        part(s["prefix_table"], s["prefix_lens"].long(), edges[:-1], edges[1:] - edges[:-1],
             max(sum(sizes["rows"][a:b]) for a, b in zip(groups, groups[1:])), False)
    logits, top = [], torch.full((total, hq), -math.inf, device="cuda")
    for table, at, there, sees in parts:
        k = _dense(s, "k", table)
        z = (_padded(s, at, there) @ k.transpose(2, 3)) * (1.0 / math.sqrt(dim))               # [groups, KV heads, rows x G, tokens]
        z = z.view(len(table), hkv, at.shape[1], hq // hkv, -1)
        z.masked_fill_(torch.arange(k.shape[2], device="cuda") >= sees[:, None, :, None, None], -math.inf)
        logits.append(z)
        m = z.amax(-1).permute(0, 2, 1, 3).reshape(*at.shape, hq)
        top[at[there]] = torch.maximum(top[at[there]], m[there])
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    weight, out = torch.zeros(total, hq, device="cuda"), torch.zeros(total, hq, dim, device="cuda")
    for (table, at, there, _), z in zip(parts, logits):
        p = torch.exp(z - base[at].view(*at.shape, hkv, -1).permute(0, 2, 1, 3)[..., None])
        o = p.flatten(2, 3) @ _dense(s, "v", table)
        weight[at[there]] += p.sum(-1).permute(0, 2, 1, 3).reshape(*at.shape, hq)[there]
        out[at[there]] += o.view(len(table), hkv, at.shape[1], -1, dim).permute(0, 2, 1, 3, 4).reshape(*at.shape, hq, dim)[there]
    s["out"].copy_(out / torch.where(weight == 0, torch.ones_like(weight), weight)[..., None])
    s["lse"].copy_(base + torch.log(weight))
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _run_own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[state["kind"]](state)


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _tokens(s, name, table_row, first, count):
    """Tokens first, ... of one sequence, [tokens, KV heads, dim], code times scale."""
    at = torch.arange(first, first + count, device="cuda")
    page, slot = table_row.long()[at // s["page"]], at % s["page"]
    pool = s[name + "_pool"]
    return pool.view(torch.int8)[page, :, slot].view(pool.dtype).double() * s[name + "_scale"][page, :, slot].double()[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    sizes = s["sizes"]
    if case["kind"] == "write":
        largest = LARGEST[case["format"]]
        pools = {name: s[name + "_pool"].double() for name in "kv"}
        scales = {name: s[name + "_scale"].double() for name in "kv"}
        cu, kept = _cu(sizes["lens"]), _cu(sizes["count"])
        for b, n in enumerate(sizes["count"]):
            src = cu[b] + (s["keep_idx"][kept[b]:kept[b + 1]].long() if "keep_idx" in s else torch.arange(n, device="cuda"))
            at = sizes["start"][b] + torch.arange(n, device="cuda")
            page, slot = s["table"][b].long()[at // case["page"]], at % case["page"]
            for name in "kv":
                x = s[name][src].double()
                top = x.abs().max(-1, keepdim=True).values
                y = torch.where(top > 0, x * largest / top.clamp(min=1e-300), torch.zeros_like(x))
                if case["format"] == "fp8":  # three bits behind the first, down to 2^-9
                    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                    y = torch.round(y / step) * step
                pools[name][page, :, slot] = torch.round(y) if case["format"] == "int8" else y
                scales[name][page, :, slot] = top[..., 0] / largest
        if case["format"] == "int8":
            pools = {name: p.to(torch.int8) for name, p in pools.items()}
        return {"k": pools["k"], "v": pools["v"], "k_scale": scales["k"], "v_scale": scales["v"]}
    if case["kind"] == "read":
        return {name: torch.cat([_tokens(s, name, s["table"][b], a, n) for b, (a, n) in enumerate(zip(sizes["start"], sizes["lens"]))]) for name in "kv"}
    group = s["hq"] // s["hkv"]
    cu, edges = _cu(sizes["rows"]), sizes["cu_prefix"]
    outs, lses = [], []
    for b, (n, r) in enumerate(zip(sizes["lens"], sizes["rows"])):
        k, v = _tokens(s, "k", s["table"][b], 0, n), _tokens(s, "v", s["table"][b], 0, n)
        hidden = torch.arange(n, device="cuda") > (n - r + torch.arange(r, device="cuda"))[:, None]
        for g, p in enumerate(sizes["prefix_lens"]):
            if edges[g] <= b < edges[g + 1]:
                k = torch.cat([_tokens(s, "k", s["prefix_table"][g], 0, p), k])
                v = torch.cat([_tokens(s, "v", s["prefix_table"][g], 0, p), v])
                hidden = torch.cat([torch.zeros(r, p, dtype=torch.bool, device="cuda"), hidden], 1)
        q = s["q"][cu[b]:cu[b + 1]].double()
        o, l = torch.empty_like(q), torch.empty(r, s["hq"], dtype=torch.float64, device="cuda")
        for h in range(s["hq"]):
            z = (q[:, h] @ k[:, h // group].T / math.sqrt(s["dim"])).masked_fill(hidden, -math.inf)
            l[:, h] = torch.logsumexp(z, 1)
            o[:, h] = torch.exp(z - l[:, h, None]) @ v[:, h // group]
        outs.append(o)
        lses.append(l)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    s = _sizes(case)
    if case["kind"] != "attend":  # K and V: a row in bf16 on one side, a code per value and a scale on the other
        rows = sum(s["count"])
        return {"bytes": rows * hkv * 2 * (3 * dim + 4) + (4 * rows if case.get("keep_lo") else 0), "flops": 0}
    rows = sum(s["rows"])
    tokens = sum(s["lens"]) + sum(s["prefix_lens"])  # a shared prefix is read once
    seen = sum(r * (n - r) + r * (r + 1) // 2 for r, n in zip(s["rows"], s["lens"]))
    for a, b, p in zip(s["cu_prefix"], s["cu_prefix"][1:], s["prefix_lens"]):
        seen += p * sum(s["rows"][a:b])
    return {"bytes": tokens * hkv * 2 * (dim + 4) + rows * hq * (4 * dim + 4), "flops": 4.0 * seen * hq * dim}
