"""The work around the 8-bit K/V cache as measurable cases: queries and keys normed per head and rotated by positions on one or three axes,
the same for new tokens straight into the cache's pages, attention weights summed up per cached token, and eviction of the lightest.

Sizes are those of the package's workloads (``workloads.py``), or generic ones of the same kind; ``draw`` spreads over the same ranges.
Values are made on the GPU from the seed: positions as audio-visual prompts have them (text, then frames of a grid), keys with a per-token
component along a direction that all query rows share, attention weights with a heavy tail and exact zeros.
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
EPS = 1e-6
BASE = 1e6          # of the rotation's frequencies
GRID = 16           # a frame is GRID x GRID tokens

LARGEST = {"int8": 127.0, "fp8": 448.0}  # a row's largest magnitude is laid on this code


def _case(name, kind, shape, **more):
    hq, hkv, dim = shape
    c = {"kind": kind, "q_heads": hq, "kv_heads": hkv, "dim": dim, **more}
    return {"name": name, **c} if name else c


def _rotate(name, shape, tokens, axes, rotary, norm, interleaved=False, packed=True):
    return _case(name, "rotate", shape, tokens=tokens, axes=axes, rotary=rotary, norm=norm, interleaved=interleaved, packed=packed)


def _write(name, shape, fmt, page, batch, lo, hi, start_hi, axes, rotary, norm, layout, interleaved=False, packed=True):
    """`lo`..`hi` new tokens of each sequence; `start_hi`: most tokens that a sequence has in the cache before."""
    return _case(name, "write", shape, format=fmt, page=page, batch=batch, lo=lo, hi=hi, start_hi=start_hi, axes=axes, rotary=rotary, norm=norm,
                 interleaved=interleaved, packed=packed, layout=layout)


def _weigh(name, shape, fmt, page, batch, lo, hi, rows_lo, rows_hi, causal, decay, fresh, layout):
    """`lo`..`hi` tokens of a sequence, `rows_lo`..`rows_hi` query rows; `fresh`: as many of the last tokens have no weight yet."""
    return _case(name, "weigh", shape, format=fmt, page=page, batch=batch, lo=lo, hi=hi, rows_lo=rows_lo, rows_hi=rows_hi, causal=causal, decay=decay,
                 fresh=fresh, layout=layout)


def _evict(name, shape, fmt, page, batch, lo, hi, keep_lo, keep_hi, first, recent, joint, layout):
    return _case(name, "evict", shape, format=fmt, page=page, batch=batch, lo=lo, hi=hi, keep_lo=keep_lo, keep_hi=keep_hi, first=first, recent=recent,
                 joint=joint, layout=layout)


def listed():
    return [
        # a layer's queries and keys of four long clips, positions (time, height, width)
        _rotate("rotate_4x16384", MISTRAL, 65536, 3, 128, False),
        # one prompt's, normed per head
        _rotate("rotate_norm_2230", QWEN2, 2230, 3, 128, True),
        # one decoding step of 32 sequences, normed, pairs of neighbours (latency)
        _rotate("rotate_norm_32", QWEN2, 32, 1, 128, True, interleaved=True, packed=False),
        # one decoding step of 32 sequences, straight into the cache (latency)
        _write("write_token_32", QWEN2, "fp8", 16, 32, 1, 1, 4096, 3, 128, True, 1),
        # a few drafted tokens each of eight sequences of a small decoder, half of each head rotated
        _write("write_drafts_8", TINY, "fp8", 32, 8, 2, 8, 744, 1, 32, False, 2, interleaved=True),
        # a ragged batch of short prompts that are not pruned; int8 codes are read back, as the prompt's own attention takes them
        _write("write_prompts_16", MISTRAL, "int8", 64, 16, 300, 1500, 0, 3, 128, True, 3),
        # the attention that 32 ragged sequences' next tokens pay, added to what they have
        _weigh("weigh_answer_ragged_32", QWEN2, "fp8", 64, 32, 512, 4096, 1, 1, True, 1.0, 1, 4),
        # ... that the next tokens of four long clips pay, older weights fading
        _weigh("weigh_answer_4x16384", MISTRAL, "int8", 256, 4, 16384, 16384, 1, 1, True, 0.98, 1, 5),
        # all tokens of 16 questions on the one long clip that they share (the largest)
        _weigh("weigh_questions_on_16384", MISTRAL, "int8", 64, 1, 16384, 16384, 1536, 1536, False, 1.0, 0, 6),
        # one short sequence loses a fifth (latency)
        _evict("evict_1x1024", QWEN2, "int8", 64, 1, 1024, 1024, 0.8, 0.8, 4, 64, False, 7),
        # 32 ragged sequences, each head on its own, to pages of their own
        _evict("evict_ragged_32", QWEN2, "fp8", 32, 32, 512, 4096, 0.3, 0.7, 4, 128, False, 8),
        # four long clips, one set of tokens for all heads
        _evict("evict_joint_4x16384", MISTRAL, "int8", 64, 4, 16384, 16384, 0.4, 0.4, 16, 256, True, 9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotate", "write", "weigh", "weigh", "evict", "evict"))
    shape, fmt, page, layout = rng.choice(SHAPES), rng.choice(("int8", "fp8")), rng.choice((16, 32, 64, 128, 256)), rng.randrange(1 << 20)
    turn = dict(axes=rng.choice((1, 3)), rotary=rng.choice((shape[2], shape[2], shape[2] // 2)), norm=rng.random() < 0.5,
                interleaved=rng.random() < 0.3, packed=rng.random() < 0.6)
    if kind == "rotate":
        return _rotate("", shape, _log_int(rng, 1, 65536), **turn)
    if kind == "write":
        total = _log_int(rng, 1, 16384)
        batch = min(_log_int(rng, 1, 64), total)
        hi = max(1, total // batch)
        return _write("", shape, fmt, page, batch, max(1, int(hi * rng.uniform(0.2, 1.0))), hi, rng.choice((0, _log_int(rng, 1, 2000))), layout=layout, **turn)
    batch = _log_int(rng, 1, 64)
    hi = _log_int(rng, 60, 16384)
    batch = min(batch, max(1, 131072 // hi))
    if kind == "evict":
        keep = round(rng.uniform(0.2, 0.95), 3)
        return _evict("", shape, fmt, page, batch, max(1, int(hi * rng.uniform(0.2, 1.0))), hi, max(0.05, keep - 0.2), keep, rng.choice((0, 4, 16)),
                      rng.choice((0, 32, 200)), rng.random() < 0.3, layout)
    rows_hi = min(hi, rng.choice((1, 1, _log_int(rng, 2, 8), _log_int(rng, 9, 128), _log_int(rng, 129, 1000))))
    batch = max(1, min(batch, (1 << 29) // (rows_hi * shape[0] * hi)))
    return _weigh("", shape, fmt, page, batch, max(rows_hi, int(hi * rng.uniform(0.2, 1.0))), hi, max(1, int(rows_hi * rng.uniform(0.2, 1.0))), rows_hi,
                  rng.random() < 0.7, rng.choice((1.0, 0.98, 0.0)), rng.choice((0, rows_hi)), layout)


# ---- sizes (a case fixes them; only the values come from the seed) -----------------------------------

def _sizes(case):
    if case["kind"] == "rotate":
        return {"lens": [case["tokens"]]}
    rng = random.Random(case["layout"])
    n = [rng.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]
    s = {"lens": n}
    if case["kind"] == "write":
        s["start"] = [rng.randint(0, case["start_hi"]) for _ in n]
    elif case["kind"] == "weigh":
        s["rows"] = [min(m, rng.randint(case["rows_lo"], case["rows_hi"])) for m in n]
    else:
        s["keep"] = [max(1, int(m * rng.uniform(case["keep_lo"], case["keep_hi"]))) for m in n]
    return s


def _cu(counts):
    cu = [0]
    for c in counts:
        cu.append(cu[-1] + c)
    return cu


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(case):
    return [BASE ** (-2.0 * i / case["rotary"]) for i in range(case["rotary"] // 2)]


def _axes(case):
    """Which axis turns each pair: a quarter of them time, then three eighths each height and width."""
    pairs = case["rotary"] // 2
    if case["axes"] == 1:
        return [0] * pairs
    return [0 if 4 * i < pairs else 1 if 8 * i < 5 * pairs else 2 for i in range(pairs)]


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
    """Page table [sequences, most pages] for sequences of that many tokens, pages in no order; -1 where a sequence has none."""
    need = [-(-n // case["page"]) for n in tokens]
    ids = used + torch.randperm(sum(need), generator=gen, device="cuda")
    table = torch.full((len(need), max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    cu = _cu(need)
    for b, m in enumerate(need):
        table[b, :m] = ids[cu[b]:cu[b + 1]]
    return table, used + sum(need)


def _pool(case, pages):
    """Pools [pages, KV heads, page tokens, dim] and scales without the last, zero."""
    code = torch.int8 if case["format"] == "int8" else torch.float8_e4m3fn
    shape = (pages, case["kv_heads"], case["page"])
    new = lambda: torch.zeros(*shape, case["dim"], dtype=torch.int8, device="cuda").view(code)  # noqa: E731
    return {"k_pool": new(), "v_pool": new(), "k_scale": torch.zeros(shape, device="cuda"), "v_scale": torch.zeros(shape, device="cuda")}


def _spread(counts):
    """Of packed rows: the sequence, and the place in it."""
    b = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).cuda()
    return b, torch.arange(sum(counts), device="cuda") - _int(_cu(counts)).long()[b]


def _fill(case, state, name, table, lens, x):
    b, i = _spread(lens)
    to, slot = table[b, i // case["page"]].long(), i % case["page"]
    c, s = _codes(case, x)
    state[name + "_pool"].view(torch.int8)[to, :, slot] = c.view(torch.int8)
    state[name + "_scale"][to, :, slot] = s


def _positions(gen, case, total):
    """[axes, tokens]: a clip somewhere in a long conversation; frames of a grid behind one another."""
    at = torch.randint(0, 100000, (1,), generator=gen, device="cuda")
    i = torch.arange(total, device="cuda")
    t, h, w = i // (GRID * GRID), i // GRID % GRID, i % GRID
    pos = (torch.stack([t, h, w]) if case["axes"] == 3 else i[None]) + at
    return pos.to(torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, dim, kind = case["q_heads"], case["kv_heads"], case["dim"], case["kind"]
    s = _sizes(case)
    state = {"kind": kind, "hkv": hkv, "hq": hq, "dim": dim, "sizes": s, "case": case}
    normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    if kind in ("rotate", "write"):
        total = sum(s["lens"])
        if case["packed"]:
            whole = normal(total, hq + 2 * hkv, dim).to(torch.bfloat16)
            state.update(q=whole[:, :hq], k=whole[:, hq:hq + hkv], v=whole[:, hq + hkv:])
        else:
            state.update(q=normal(total, hq, dim).to(torch.bfloat16), k=normal(total, hkv, dim).to(torch.bfloat16), v=normal(total, hkv, dim).to(torch.bfloat16))
        state.update(pos=_positions(gen, case, total), q_out=torch.empty(total, hq, dim, dtype=torch.bfloat16, device="cuda"),
                     frequencies=_frequencies(case), axis=_axes(case), freq_gpu=torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda"),
                     axis_gpu=_int(_axes(case)).long(), rotary=case["rotary"], interleaved=case["interleaved"])
        state["q_norm"], state["k_norm"] = ((1 + 0.1 * normal(dim)).to(torch.bfloat16) for _ in "qk") if case["norm"] else (None, None)
        new = lambda: torch.empty(total, hkv, dim, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        if kind == "rotate":
            return {**state, "k_out": new()}
        table, pages = _tables(gen, case, [a + n for a, n in zip(s["start"], s["lens"])])
        b, i = _spread(s["lens"])
        state.update(_pool(case, pages), table=table, start=_int(s["start"]), cu_seqlens=_int(_cu(s["lens"])), page=case["page"], format=case["format"],
                     token_seq=b, token_at=i + _int(s["start"]).long()[b], k_read=new(), v_read=new())
        return state
    state.update(page=case["page"], format=case["format"])
    lens = s["lens"]
    table, pages = _tables(gen, case, lens)
    if kind == "evict":
        state["out_table"], pages = _tables(gen, case, s["keep"], pages)
        state.update(_pool(case, pages), table=table, kv_lens=_int(lens), keep_counts=_int(s["keep"]), lens_out=torch.zeros(len(lens), dtype=torch.int32, device="cuda"),
                     keep_idx=torch.zeros(len(lens), hkv, max(s["keep"]), dtype=torch.int32, device="cuda"), kept_seq_at=_spread(s["keep"]))
        for name in "kv":
            _fill(case, state, name, table, lens, normal(sum(lens), hkv, dim))
        state["weights"] = torch.exp(2 * normal(*state["k_scale"].shape)) * (torch.rand(state["k_scale"].shape, generator=gen, device="cuda") > 0.05)
        return state
    shared = normal(hkv, dim)
    rows = s["rows"]
    q = normal(sum(rows), hkv, hq // hkv, dim) * math.sqrt(1 - SHARED ** 2) + SHARED * shared[:, None, :]
    state.update(_pool(case, pages), table=table, kv_lens=_int(lens), q=q.reshape(sum(rows), hq, dim).to(torch.bfloat16), cu_qlens=_int(_cu(rows)),
                 causal=case["causal"], decay=case["decay"])
    _fill(case, state, "k", table, lens, torch.cat([_keys(gen, case, n, shared) for n in lens]))
    state["weights"] = torch.exp(normal(*state["k_scale"].shape)) * (sum(rows) * (hq // hkv) / sum(lens))  # about what one more call adds
    state["weighed_lens"] = _int([max(0, n - case["fresh"]) for n in lens]) if case["fresh"] else None
    state["row_seq_at"] = _spread(rows)
    z, _, _ = _logits(state)
    state["lse"] = torch.logsumexp(z, -1)[state["row_seq_at"][0], :, state["row_seq_at"][1]].reshape(sum(rows), hq).contiguous()
    return state


# ---- the framework's operators -------------------------------------------------------------------------

def _handle(state):
    """What a program makes once: the cache's handle, parameters, workspace."""
    if "F" not in state:
        from paper_2601_13143_b200 import fastav as F
        s, case = state["sizes"], state["case"]
        if state["kind"] != "rotate":
            state["cache"] = F.KvCache(state["k_pool"], state["v_pool"], state["k_scale"], state["v_scale"])
        if state["kind"] in ("rotate", "write"):
            state["params"] = F.make_rotate_params(batch=len(s["lens"]), q=state["q"], k=state["k"], v=state["v"], q_out=state["q_out"], k_out=state.get("k_out"),
                                                   pos=state["pos"], frequencies=state["frequencies"], axis=state["axis"], interleaved=case["interleaved"],
                                                   norm_eps=EPS)
            if state["kind"] == "write":
                state["read_params"] = F.make_params(batch=len(s["lens"]), total_tokens=sum(s["lens"]), max_seqlen=max(s["lens"]), total_q=0, max_qlen=0, total_keep=0,
                                                     max_keep=0, num_q_heads=state["hq"], num_kv_heads=state["hkv"], head_dim=state["dim"], hidden=0,
                                                     k_out=state["k_read"], v_out=state["v_read"])
        elif state["kind"] == "weigh":
            state["params"] = F.make_attend_params(batch=len(s["lens"]), total_q=sum(s["rows"]), max_qlen=max(s["rows"]), num_q_heads=state["hq"],
                                                   max_kv_len=max(s["lens"]), q=state["q"], out=state["q"], page_table=state["table"],
                                                   flags=F.FASTAV_CAUSAL if case["causal"] else 0)
        else:
            state["params"] = F.make_evict_params(batch=len(s["lens"]), max_kv_len=max(s["lens"]), max_keep=max(s["keep"]), page_table=state["table"],
                                                  out_table=state["out_table"], first=case["first"], recent=case["recent"],
                                                  flags=F.FASTAV_EVICT_JOINT if case["joint"] else 0)
            state["workspace"] = torch.empty(F.fastav_evict_workspace_bytes(state["params"], state["cache"]), dtype=torch.uint8, device="cuda")
        state["F"] = F
    return state["F"], state["params"]


def _run_own(s):
    F, params = _handle(s)
    if s["kind"] == "rotate":
        F.fastav_rotate(params, s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], s["q_norm"], s["k_norm"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if s["kind"] == "write":
        F.fastav_rotate_write(params, s["cache"], s["q"], s["k"], s["v"], s["pos"], s["cu_seqlens"], s["table"], s["start"], s["q_out"], s["q_norm"], s["k_norm"])
        if s["format"] == "int8":
            F.fastav_cache_read(s["read_params"], s["cache"], s["table"], s["start"], s["cu_seqlens"], s["k_read"], s["v_read"])
            return {"q": s["q_out"], "k": s["k_read"], "v": s["v_read"]}
        return _written(s)
    if s["kind"] == "weigh":
        F.fastav_cache_weigh(params, s["cache"], s["weights"], s["q"], s["lse"], s["cu_qlens"], s["table"], s["kv_lens"], s["weighed_lens"], s["decay"])
        return {"weights": s["weights"]}
    F.fastav_cache_evict(params, s["cache"], s["weights"], s["table"], s["kv_lens"], s["keep_counts"], s["lens_out"], s["workspace"], s["out_table"], s["keep_idx"])
    return _evicted(s)


# ---- their plain forms -----------------------------------------------------------------------------------

def _written(s):
    """e4m3 codes are the values of their type, in units of the scales."""
    return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _evicted(s):
    """The whole cache (int8 codes are whole numbers, moved as they are), every survivor's weight and where it was."""
    return {"k": s["k_pool"], "v": s["v_pool"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "weights": s["weights"], "lens": s["lens_out"], "idx": s["keep_idx"]}


def _turned(s, x, norm):
    """x [tokens, heads, dim] normed and rotated, in fp32; the angles in 64 bits."""
    x = x.float()
    if norm is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * norm.float()
    angle = s["pos"].double()[s["axis_gpu"]].T * s["freq_gpu"]      # [tokens, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    r = s["rotary"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    both = (a * cos - b * sin, a * sin + b * cos)
    both = torch.stack(both, -1).flatten(-2) if s["interleaved"] else torch.cat(both, -1)
    return torch.cat([both, x[..., r:]], -1)


def _plain_rotate(s):
    s["q_out"].copy_(_turned(s, s["q"], s["q_norm"]))
    s["k_out"].copy_(_turned(s, s["k"], s["k_norm"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _plain_put(s, name, x):
    """Rows x into the pages; (codes, scales) as written."""
    page, slot = s["table"][s["token_seq"], s["token_at"] // s["page"]].long(), s["token_at"] % s["page"]
    largest = LARGEST[s["format"]]
    top = x.abs().amax(-1)
    y = torch.where(top[..., None] == 0, torch.zeros_like(x), x * largest / top[..., None])
    code = y.round().clamp(-127, 127).to(torch.int8) if s["format"] == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn)
    s[name + "_pool"].view(torch.int8)[page, :, slot] = code.view(torch.int8)
    s[name + "_scale"][page, :, slot] = top / largest
    return code, top / largest


def _plain_write(s):
    s["q_out"].copy_(_turned(s, s["q"], s["q_norm"]))
    k, v = _plain_put(s, "k", _turned(s, s["k"], s["k_norm"])), _plain_put(s, "v", s["v"].float())
    if s["format"] == "int8":
        s["k_read"].copy_(k[0].float() * k[1][..., None])
        s["v_read"].copy_(v[0].float() * v[1][..., None])
        return {"q": s["q_out"], "k": s["k_read"], "v": s["v_read"]}
    return _written(s)


def _logits(s):
    """[sequences, heads, most rows, most tokens] in fp32, -inf where a row does not see the token; and of the tokens their pages and places."""
    lens, rows, cu = s["kv_lens"].long(), (s["cu_qlens"][1:] - s["cu_qlens"][:-1]).long(), s["cu_qlens"].long()
    most, most_rows, hkv = max(s["sizes"]["lens"]), max(s["sizes"]["rows"]), s["hkv"]
    i, r = torch.arange(most, device="cuda"), torch.arange(most_rows, device="cuda")
    page, slot = s["table"].clamp(min=0).long()[:, i // s["page"]], (i % s["page"]).expand(len(lens), -1)
    k = s["k_pool"].view(torch.int8)[page, :, slot].view(s["k_pool"].dtype).float() * s["k_scale"][page, :, slot][..., None]   # [sequences, tokens, heads, dim]
    q = s["q"].float()[(cu[:-1, None] + r).clamp(max=len(s["q"]) - 1)]                                                       # [sequences, rows, heads, dim]
    q = q.view(len(lens), most_rows, hkv, -1, s["dim"]).permute(0, 2, 3, 1, 4).flatten(2, 3)
    z = (q @ k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(s["dim"]))
    z = z.view(len(lens), s["hq"], most_rows, most)
    sees = (lens[:, None] - rows[:, None] + r + 1 if s["causal"] else lens[:, None].expand(-1, most_rows)) * (r < rows[:, None])
    return z.masked_fill_(i >= sees[:, None, :, None], -math.inf), page, slot


def _plain_weigh(s):
    z, page, slot = _logits(s)
    b, r = s["row_seq_at"]
    lse = torch.full(z.shape[:3], math.inf, device="cuda")
    lse[b, :, r] = s["lse"]
    paid = z.sub_(lse[..., None]).exp_().sum(2).view(len(z), s["hkv"], -1, z.shape[-1]).sum(2).transpose(1, 2)                 # [sequences, tokens, heads]
    i = torch.arange(z.shape[-1], device="cuda")
    before = s["weights"][page, :, slot]
    if s["weighed_lens"] is not None:
        before = before * (i < s["weighed_lens"][:, None])[..., None]
    there = i < s["kv_lens"][:, None]
    s["weights"][page[there], :, slot[there]] = (s["decay"] * before + paid)[there]
    return {"weights": s["weights"]}


def _plain_evict(s):
    lens, keep, case = s["kv_lens"].long(), s["keep_counts"].long(), s["case"]
    most, most_kept = max(s["sizes"]["lens"]), max(s["sizes"]["keep"])
    i = torch.arange(most, device="cuda")
    page, slot = s["table"].clamp(min=0).long()[:, i // s["page"]], (i % s["page"]).expand(len(lens), -1)
    w = s["weights"][page, :, slot].transpose(1, 2)                       # [sequences, heads, tokens]
    if case["joint"]:
        w = w.double().sum(1, keepdim=True).float().expand(-1, s["hkv"], -1)
    stays = (i < case["first"]) | (i >= lens[:, None] - case["recent"])
    w = w.masked_fill(stays[:, None], math.inf).masked_fill((i >= lens[:, None])[:, None], -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :most_kept]
    chosen = order.masked_fill(torch.arange(most_kept, device="cuda") >= keep[:, None, None], most).sort(-1).values
    b, r = s["kept_seq_at"]
    src = chosen[b, :, r]                                                 # [kept, heads]
    h = torch.arange(s["hkv"], device="cuda")
    src_page, dst_page = s["table"][b[:, None], src // s["page"]].long(), s["out_table"][b, r // s["page"]].long()[:, None]
    at, to = (src_page, h, src % s["page"]), (dst_page, h, (r % s["page"])[:, None])
    s["k_pool"].view(torch.int8)[to] = s["k_pool"].view(torch.int8)[at]
    s["v_pool"].view(torch.int8)[to] = s["v_pool"].view(torch.int8)[at]
    s["k_scale"][to], s["v_scale"][to], s["weights"][to] = s["k_scale"][at], s["v_scale"][at], s["weights"][at]
    s["lens_out"].copy_(torch.minimum(keep, lens))
    s["keep_idx"][b, :, r] = src.to(torch.int32)
    return _evicted(s)


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _plain_rotate, "write": _plain_write, "weigh": _plain_weigh, "evict": _plain_evict}[state["kind"]](state)


# ---- the definition in 64 bits ---------------------------------------------------------------------------

def _exact_turned(case, s, x, norm):
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * norm.double()
    y = x.clone()
    half = case["rotary"] // 2
    for i, (f, axis) in enumerate(zip(_frequencies(case), _axes(case))):
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half)
        turn = s["pos"][axis].double()[:, None] * f
        y[..., a] = x[..., a] * torch.cos(turn) - x[..., b] * torch.sin(turn)
        y[..., b] = x[..., b] * torch.cos(turn) + x[..., a] * torch.sin(turn)
    return y


def _exact_codes(case, x):
    largest = LARGEST[case["format"]]
    top = x.abs().max(-1, keepdim=True).values
    y = torch.where(top > 0, x * largest / top.clamp(min=1e-300), torch.zeros_like(x))
    if case["format"] == "int8":
        return torch.round(y), top / largest
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)  # three bits behind the first, down to 2^-9
    return torch.round(y / step) * step, top / largest


def exact(case, seed):
    s = prepare(case, seed)
    sizes, page = s["sizes"], case.get("page")
    where = lambda table, first, count: (table.long()[torch.arange(first, first + count, device="cuda") // page],  # noqa: E731
                                         torch.arange(first, first + count, device="cuda") % page)
    if case["kind"] == "rotate":
        return {"q": _exact_turned(case, s, s["q"], s["q_norm"]), "k": _exact_turned(case, s, s["k"], s["k_norm"])}
    if case["kind"] == "write":
        q = _exact_turned(case, s, s["q"], s["q_norm"])
        k, v = _exact_codes(case, _exact_turned(case, s, s["k"], s["k_norm"])), _exact_codes(case, s["v"].double())
        if case["format"] == "int8":
            return {"q": q, "k": k[0] * k[1], "v": v[0] * v[1]}
        got = {"q": q, "k": s["k_pool"].double(), "v": s["v_pool"].double(), "k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double()}
        cu = _cu(sizes["lens"])
        for b, (first, n) in enumerate(zip(sizes["start"], sizes["lens"])):
            to, slot = where(s["table"][b], first, n)
            for name, (c, scale) in (("k", k), ("v", v)):
                got[name][to, :, slot] = c[cu[b]:cu[b + 1]]
                got[name + "_scale"][to, :, slot] = scale[cu[b]:cu[b + 1], :, 0]
        return got
    if case["kind"] == "weigh":
        group, cu, weights = s["hq"] // s["hkv"], _cu(sizes["rows"]), s["weights"].double()
        for b, (n, rows) in enumerate(zip(sizes["lens"], sizes["rows"])):
            to, slot = where(s["table"][b], 0, n)
            old = max(0, n - case["fresh"])
            paid = torch.zeros(n, s["hkv"], dtype=torch.float64, device="cuda")
            hidden = torch.arange(n, device="cuda") > (n - rows + torch.arange(rows, device="cuda"))[:, None]
            for h in range(s["hq"]):
                k = s["k_pool"].view(torch.int8)[to, h // group, slot].view(s["k_pool"].dtype).double() * s["k_scale"][to, h // group, slot].double()[:, None]
                z = s["q"][cu[b]:cu[b + 1], h].double() @ k.T / math.sqrt(s["dim"]) - s["lse"][cu[b]:cu[b + 1], h].double()[:, None]
                paid[:, h // group] += torch.exp(z.masked_fill(hidden, -math.inf) if case["causal"] else z).sum(0)
            paid[:old] += case["decay"] * s["weights"][to[:old], :, slot[:old]].double()
            weights[to, :, slot] = paid
        return {"weights": weights}
    got = {"k": s["k_pool"].view(torch.int8).clone(), "v": s["v_pool"].view(torch.int8).clone(), "k_scale": s["k_scale"].double(),
           "v_scale": s["v_scale"].double(), "weights": s["weights"].double(), "lens": s["lens_out"], "idx": s["keep_idx"]}
    for b, (n, kept) in enumerate(zip(sizes["lens"], sizes["keep"])):
        at, slot = where(s["table"][b], 0, n)
        to, to_slot = where(s["out_table"][b], 0, kept)
        w = s["weights"][at, :, slot].double()
        if case["joint"]:
            w = w.sum(1, keepdim=True).expand(-1, s["hkv"]).float().double()
        w = w.clone()
        w[:case["first"]] = math.inf
        w[max(0, n - case["recent"]):] = math.inf
        for h in range(s["hkv"]):
            chosen = torch.argsort(-w[:, h], stable=True)[:kept].sort().values
            for name, pool in (("k", s["k_pool"].view(torch.int8)), ("v", s["v_pool"].view(torch.int8)), ("k_scale", s["k_scale"]), ("v_scale", s["v_scale"]),
                               ("weights", s["weights"])):
                got[name][to, h, to_slot] = pool[at[chosen], h, slot[chosen]].to(got[name].dtype)
            got["idx"][b, h, :kept] = chosen.to(torch.int32)
        got["lens"][b] = min(n, kept)
    if case["format"] == "fp8":
        got["k"], got["v"] = (got[name].view(torch.float8_e4m3fn).double() for name in "kv")
    return got


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    hq, hkv, dim = case["q_heads"], case["kv_heads"], case["dim"]
    s = _sizes(case)
    tokens = sum(s["lens"])
    if case["kind"] in ("rotate", "write"):
        flops = tokens * (hq + hkv) * (3.0 * case["rotary"] + (4 * dim if case["norm"] else 0))
        inputs = tokens * ((hq + hkv) * 2 * dim + 4 * case["axes"])
        if case["kind"] == "rotate":
            return {"bytes": inputs + tokens * (hq + hkv) * 2 * dim, "flops": flops}
        back = tokens * hkv * 2 * (3 * dim + 4) if case["format"] == "int8" else 0   # codes and scales read, bf16 written
        return {"bytes": inputs + tokens * (hq * 2 * dim + hkv * 2 * dim + 2 * hkv * (dim + 4)) + back, "flops": flops}
    if case["kind"] == "weigh":
        rows = sum(s["rows"])
        seen = sum(r * (n - r) + r * (r + 1) // 2 if case["causal"] else r * n for r, n in zip(s["rows"], s["lens"]))
        return {"bytes": tokens * hkv * (dim + 4 + 8) + rows * hq * (2 * dim + 4), "flops": 2.0 * seen * hq * dim}
    kept = sum(s["keep"])
    return {"bytes": tokens * hkv * 4 + kept * hkv * (4 * (dim + 4) + 4 + 4), "flops": 0}
