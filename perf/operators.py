"""Workloads of the key/value cache operators: appending to a cache held in 8 bits, attention over
it, and eviction by accumulated attention weight.

The cache is a pool of blocks.  `codes` int8 [blocks][2][kv_heads][block][dim] holds keys (0) and
values (1), `scales` float32 [blocks][2][kv_heads] one scale for each block of tokens and head; an
element is code * scale.  `score` float32 [blocks][kv_heads][block] holds the attention weight that
each cached token has gathered.  `table` int32 [batch][max_blocks] names the blocks of a sequence,
`lens` int32 [batch] its tokens, and `starts` int32 [batch + 1] the rows of the new tokens, which
are the last of their sequence.

Every case runs in two forms: elementary torch operations in float32 (`own` false), or the calls
that a program makes of the library (`own` true).
"""
import math

import torch

own = False

PHI = 0.6180339887498949


def listed():
    def case(name, op, batch, heads, kv_heads, dim, block, length, new, ragged, scores=False, budget=0, recent=0):
        return {"name": name, "op": op, "batch": batch, "heads": heads, "kv_heads": kv_heads, "dim": dim, "block": block,
                "len": length, "new": new, "ragged": ragged, "scores": scores, "budget": budget, "recent": recent}

    return [
        # one generated token of each of 24 LLaMA-7B conversations enters the cache
        case("append_decode", "append", 24, 32, 32, 128, 64, 2047, 1, True),
        # three LLaMA-7B prompts of different lengths enter an empty cache
        case("append_prompt", "append", 3, 32, 32, 128, 64, 4093, 0, True),
        # the smallest call: one LLaMA-7B user, a short conversation, one token
        case("decode_single", "attention", 1, 32, 32, 128, 64, 333, 1, False),
        # a LLaMA-7B server's step over conversations of very different lengths
        case("decode_batch", "attention", 32, 32, 32, 128, 64, 4096, 1, True),
        # grouped key heads over a very long document, with the weights gathered for an eviction
        case("decode_long", "attention", 2, 64, 8, 128, 128, 100003, 1, True, True),
        # LLaMA-13B checking five drafted tokens of each conversation, small blocks
        case("decode_draft", "attention", 8, 40, 40, 128, 16, 1777, 5, True),
        # a small grouped-head model, 64-wide heads, weights gathered at every step
        case("decode_scores", "attention", 48, 32, 8, 64, 32, 3001, 1, True, True),
        # one LLaMA-7B prompt from its first token
        case("prompt", "attention", 1, 32, 32, 128, 64, 4096, 0, False),
        # the next 700 tokens of two long prompts, grouped heads of 64, with the weights gathered
        case("prompt_chunk", "attention", 2, 32, 8, 64, 128, 12345, 700, True, True),
        # LLaMA-13B prompts of different lengths, with the weights gathered for an eviction
        case("prompt_ragged", "attention", 4, 40, 40, 128, 32, 1500, 0, True, True),
        # eight LLaMA-7B conversations shortened to a quarter
        case("evict_batch", "evict", 8, 32, 32, 128, 64, 8000, 0, True, False, 2048, 256),
        # a very long document with grouped key heads shortened to a budget that ends inside a block
        case("evict_long", "evict", 1, 64, 8, 128, 128, 100003, 0, False, False, 12300, 1000),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    dim = rng.choice([64, 128, 128])
    heads, kv_heads = rng.choice([(32, 32), (40, 40), (32, 8), (64, 8), (40, 10), (16, 2), (8, 1), (64, 64)])
    c = {"op": rng.choice(["append", "attention", "attention", "attention", "evict"]), "heads": heads, "kv_heads": kv_heads,
         "dim": dim, "block": rng.choice([16, 32, 64, 64, 128]), "ragged": rng.random() < 0.7, "scores": False,
         "budget": 0, "recent": 0}
    if c["op"] == "append":
        if rng.random() < 0.5:      # generated tokens
            c.update(batch=_log_uniform(rng, 1, 64), new=rng.choice([1, 1, 2, 5]))
            c["len"] = _log_uniform(rng, 20, max(40, 2000000 // (c["batch"] * kv_heads)))
        else:                       # prompts, or pieces of them
            c["new"] = _log_uniform(rng, 17, 3000)
            c["len"] = c["new"] + (0 if rng.random() < 0.5 else _log_uniform(rng, 1, 3000))
            c["batch"] = max(1, min(_log_uniform(rng, 1, 8), 250000 // (c["new"] * kv_heads)))
    elif c["op"] == "attention":
        c["scores"] = rng.random() < 0.4
        if rng.random() < 0.65:     # generated or drafted tokens
            c.update(batch=_log_uniform(rng, 1, 64), new=rng.choice([1, 1, 1, 2, 4, 7]))
            c["len"] = _log_uniform(rng, 40, max(80, min(100000, 2300000 // (c["batch"] * kv_heads))))
        else:
            c["new"] = _log_uniform(rng, 30, 3000)
            c["len"] = c["new"] + (0 if rng.random() < 0.5 else _log_uniform(rng, 1, 6000))
            c["batch"] = max(1, min(_log_uniform(rng, 1, 6), int(3.5e8 / (c["new"] * c["len"] * heads))))
    else:
        c["batch"] = _log_uniform(rng, 1, 16)
        c["len"] = _log_uniform(rng, 300, max(600, min(100000, 1800000 // (c["batch"] * kv_heads))))
        c["budget"] = max(16, int(c["len"] * rng.uniform(0.05, 0.6)))
        c["recent"] = int(c["budget"] * rng.uniform(0.0, 0.5))
        c["new"] = 0
    return c


def _sizes(case):
    """(lens, new): tokens and new tokens of each sequence."""
    lens = [case["len"]] * case["batch"]
    if case["ragged"]:
        lens = [max(1, int(case["len"] * (1.0 - 0.9 * ((b * PHI) % 1.0)))) for b in range(case["batch"])]
    new = [min(n, case["new"]) if case["new"] else n for n in lens]
    return lens, new


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens, new = _sizes(case)
    B, H, KH, D, T = (case[k] for k in ("batch", "heads", "kv_heads", "dim", "block"))
    width = max(-(-n // T) for n in lens)
    kept = -(-min(case["budget"], max(lens)) // T) if case["op"] == "evict" else 0
    blocks = B * (width + kept) + 3
    order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    s = {"case": dict(case), "table": order[:B * width].view(B, width).contiguous(), "lens": dev(lens), "starts": dev(starts),
         "m": starts[-1], "max_new": max(new), "max_len": max(lens), "blocks": blocks}
    codes = torch.randn((blocks, 2, KH, T, D), generator=g, device="cuda", dtype=torch.bfloat16).mul_(36.0).round_()
    s["codes"] = codes.clamp_(-127, 127).to(torch.int8)
    spread = torch.rand((blocks, 2, KH), generator=g, device="cuda", dtype=torch.float32)
    s["scales"] = (1.0 + spread) * (1.5 / 127)
    s["score"] = torch.zeros((blocks, KH, T), dtype=torch.float32, device="cuda")
    if case["op"] == "append":
        rows = torch.randn((2, s["m"], KH, D), generator=g, device="cuda", dtype=torch.float32)
        rows[..., :: max(1, D // 4)] *= 4.0                        # a few channels of keys are always large
        s["k"], s["v"] = rows[0].bfloat16(), rows[1].bfloat16()
        # the tokens that are read back: all of every block that new tokens entered
        first = [(n - w) // T * T for n, w in zip(lens, new)]
        out = [0]
        for n, f in zip(lens, first):
            out.append(out[-1] + n - f)
        s.update(first=dev(first), out_starts=dev(out), out_m=out[-1], out_max=max(n - f for n, f in zip(lens, first)))
        s["k_out"] = torch.empty((out[-1], KH, D), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    elif case["op"] == "attention":
        s["q"] = torch.randn((s["m"], H, D), generator=g, device="cuda", dtype=torch.float32).mul_(1.4).bfloat16()
        s["softmax_scale"] = D ** -0.5
        s["out"] = torch.empty((s["m"], H, D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.empty((s["m"], H), dtype=torch.float32, device="cuda")
        if case["scores"]:
            s["score"] = torch.rand((blocks, KH, T), generator=g, device="cuda", dtype=torch.float32).mul_(0.01)
            s["score_out"] = torch.zeros_like(s["score"])
    else:
        u = torch.rand((blocks, KH, T), generator=g, device="cuda", dtype=torch.float32)
        s["score"] = 0.01 / (u + 1e-3)                             # few tokens gather much
        budget = case["budget"]
        s["dst_table"] = order[B * width:B * (width + kept)].view(B, kept).contiguous()
        s["dst_lens"] = torch.empty(B, dtype=torch.int32, device="cuda")
        s["kept"] = torch.empty((B, KH, budget), dtype=torch.int32, device="cuda")
        s["kept_lens"] = [min(n, budget) for n in lens]
        out = [0]
        for n in s["kept_lens"]:
            out.append(out[-1] + n)
        s.update(out_starts=dev(out), out_m=out[-1], out_max=max(s["kept_lens"]), first=dev([0] * B))
        s["k_out"] = torch.empty((out[-1], KH, D), dtype=torch.bfloat16, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"append": _append, "attention": _attention, "evict": _evict}[s["case"]["op"]](s)


# ---- the library's calls ------------------------------------------------------------------------
def _run_own(s):
    from paper_2309_14717_b200 import binding as Q

    c = s["case"]
    if "desc" not in s:     # made once by a program, like the buffers
        s["desc"] = Q.kv_desc(c["heads"], c["kv_heads"], c["dim"], c["block"], s["blocks"])
    d = s["desc"]
    if c["op"] == "append":
        Q.qalora_kv_append(d, s["max_new"], s["starts"], s["lens"], s["table"], s["k"], s["v"], s["codes"], s["scales"])
        Q.qalora_kv_read(d, s["out_max"], s["out_starts"], s["first"], s["table"], s["codes"], s["scales"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"], "scales": s["scales"]}
    if c["op"] == "attention":
        if "workspace" not in s:
            s["workspace"] = Q.alloc_kv_workspace(d, c["batch"], s["m"], s["max_new"], s["max_len"], c["scores"])
        score_out = s.get("score_out")
        Q.qalora_kv_attention(d, s["max_new"], s["max_len"], s["starts"], s["lens"], s["table"], s["q"], s["codes"], s["scales"],
                              s["softmax_scale"], s["out"], s["lse"], s["score"] if c["scores"] else None, score_out, s["workspace"])
        return {"out": s["out"], "lse": s["lse"], **({"score": score_out} if c["scores"] else {})}
    Q.qalora_kv_evict(d, s["max_len"], c["budget"], c["recent"], s["lens"], s["table"], s["codes"], s["scales"], s["score"],
                      s["dst_table"], s["dst_lens"], s["kept"])
    Q.qalora_kv_read(d, s["out_max"], s["out_starts"], s["first"], s["dst_table"], s["codes"], s["scales"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"], "kept": s["kept"], "lens": s["dst_lens"], "scales": s["scales"], "score": s["score"]}


# ---- elementary operations ----------------------------------------------------------------------
def _sequence_of(starts, m):
    """(sequence, place within it) of each of m rows."""
    row = torch.arange(m, device="cuda")
    b = torch.searchsorted(starts, row.to(starts.dtype), right=True) - 1
    return b, row - starts[b]


def _quantized(x, scale):
    return torch.where(scale > 0, x / scale, torch.zeros_like(x)).round().clamp(-127, 127)


def _read(s, table, m, starts, first):
    b, i = _sequence_of(starts, m)
    pos = first[b] + i
    T = s["case"]["block"]
    block, slot = table[b, pos // T].long(), pos % T
    x = s["codes"][block, :, :, slot].float() * s["scales"][block].unsqueeze(-1)
    return x[:, 0].bfloat16(), x[:, 1].bfloat16()


def _append(s):
    T, codes, scales, table, lens, starts = (s["case"]["block"], s["codes"], s["scales"], s["table"], s["lens"], s["starts"])
    b, i = _sequence_of(starts, s["m"])
    begin = lens - (starts[1:] - starts[:-1])                       # tokens before this call
    pos = begin[b] + i
    block, slot = table[b, pos // T].long(), pos % T
    x = torch.stack([s["k"], s["v"]], 1).float()                    # [m][2][kv_heads][dim]
    need = x.abs().amax(-1) / 127.0
    before = scales.clone()
    touched = scales.index_fill(0, block, 0.0)                      # blocks that begin with this call have no scale yet
    edge = table.gather(1, (begin // T).clamp(max=table.shape[1] - 1).long().unsqueeze(1)).squeeze(1).long()
    partly = (begin % T > 0) & (starts[1:] > starts[:-1])
    touched[edge] = torch.where(partly[:, None, None], before[edge], touched[edge])
    touched.scatter_reduce_(0, block[:, None, None].expand_as(need), need, "amax")
    scales.copy_(touched)
    ratio = torch.where(touched[edge] > 0, before[edge] / touched[edge], torch.zeros_like(before[edge]))
    older = partly[:, None] & (torch.arange(T, device="cuda") < (begin % T)[:, None])
    old = codes[edge].float()
    codes[edge] = torch.where(older[:, None, None, :, None], (old * ratio[..., None, None]).round(), old).to(torch.int8)
    codes[block, :, :, slot] = _quantized(x, touched[block].unsqueeze(-1)).to(torch.int8)
    k, v = _read(s, table, s["out_m"], s["out_starts"], s["first"])
    return {"k": k, "v": v, "scales": scales}


def _attention(s):
    c = s["case"]
    B, H, KH, D, T = (c[k] for k in ("batch", "heads", "kv_heads", "dim", "block"))
    G, N, table = H // KH, s["max_new"], s["table"].long()
    kv = (s["codes"][table].float() * s["scales"][table][..., None, None]).permute(2, 0, 3, 1, 4, 5)
    k, v = kv.reshape(2, B, KH, -1, D)                              # [B][kv_heads][tokens][dim]
    del kv
    new = s["starts"][1:] - s["starts"][:-1]
    b, i = _sequence_of(s["starts"], s["m"])
    q = torch.zeros((B, N, H, D), device="cuda")
    q[b, i] = s["q"].float()
    q = q.view(B, N, KH, G, D).permute(0, 2, 1, 3, 4).reshape(B, KH, N * G, D)
    pos = (s["lens"] - new)[:, None] + torch.arange(N, device="cuda")
    seen = (torch.arange(k.shape[2], device="cuda") <= pos[..., None]) & (torch.arange(N, device="cuda") < new[:, None])[..., None]
    logit = torch.matmul(q, k.transpose(2, 3)).mul_(s["softmax_scale"])
    logit = logit.view(B, KH, N, G, -1).masked_fill_(~seen[:, None, :, None], float("-inf")).view(B, KH, N * G, -1)
    top = logit.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = logit.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    share = torch.where(total > 0, 1.0 / total, torch.zeros_like(total))
    out = torch.matmul(p, v) * share
    rows = lambda x: x.reshape(B, KH, N, G, -1).permute(0, 2, 1, 3, 4).reshape(B, N, H, -1)[b, i]  # noqa: E731
    found = {"out": rows(out).bfloat16(), "lse": rows(top + total.log()).squeeze(-1)}
    if c["scores"]:
        weight = p.mul_(share).sum(2).view(B, KH, -1, T).permute(0, 2, 1, 3)       # [B][blocks][kv_heads][block]
        inside = torch.arange(weight.shape[1] * T, device="cuda").view(-1, T) < s["lens"][:, None, None]
        score = s["score_out"]
        score[table] = torch.where(inside[:, :, None], s["score"][table] + weight, score[table])
        found["score"] = score
    return found


def _evict(s):
    c = s["case"]
    B, KH, D, T, budget, recent = (c[k] for k in ("batch", "kv_heads", "dim", "block", "budget", "recent"))
    table, lens = s["table"].long(), s["lens"].long()
    score = s["score"][table].permute(0, 2, 1, 3).reshape(B, KH, -1)
    t = torch.arange(score.shape[-1], device="cuda")
    rank = torch.where((t >= (lens - recent)[:, None])[:, None], float("inf"), score)
    rank = torch.where((t < lens[:, None])[:, None], rank, float("-inf"))
    best = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :budget]
    count = lens.clamp(max=budget)
    slot = torch.arange(best.shape[-1], device="cuda")
    valid = slot < count[:, None]
    best = torch.where(valid[:, None], best, score.shape[-1]).sort(-1)[0]
    s["kept"].fill_(-1)
    s["kept"][..., :best.shape[-1]] = torch.where(valid[:, None], best, -1)
    s["dst_lens"].copy_(count)
    pad = s["dst_table"].shape[1] * T - best.shape[-1]
    best = torch.nn.functional.pad(best, (0, pad), value=score.shape[-1])           # whole blocks of the new place
    valid = torch.nn.functional.pad(valid, (0, pad), value=False)
    at = best.clamp(max=score.shape[-1] - 1)
    src = table.gather(1, (at // T).view(B, -1)).view(B, KH, -1)
    head = torch.arange(KH, device="cuda")[:, None]
    x = s["codes"][src, :, head, at % T].float() * s["scales"][src, :, head].unsqueeze(-1)   # [B][kv_heads][tokens][2][dim]
    x = torch.where(valid[:, None, :, None, None], x, torch.zeros_like(x)).view(B, KH, -1, T, 2, D)
    scale = x.abs().amax((3, 5)) / 127.0                                            # [B][kv_heads][blocks][2]
    dst = s["dst_table"].long()
    used = valid.view(B, -1, T)
    fresh = _quantized(x, scale[:, :, :, None, :, None]).to(torch.int8).permute(0, 2, 4, 1, 3, 5)
    s["codes"][dst] = torch.where(used[:, :, None, None, :, None], fresh, s["codes"][dst])
    some = used.any(-1)
    s["scales"][dst] = torch.where(some[:, :, None, None], scale.permute(0, 2, 3, 1), s["scales"][dst])
    moved = score.gather(-1, at).view(B, KH, -1, T).transpose(1, 2)
    s["score"][dst] = torch.where(used[:, :, None], moved, s["score"][dst])
    k, v = _read(s, s["dst_table"], s["out_m"], s["out_starts"], s["first"])
    return {"k": k, "v": v, "kept": s["kept"], "lens": s["dst_lens"], "scales": s["scales"], "score": s["score"]}


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    lens, new = _sizes(case)
    H, KH, D, T = (case[k] for k in ("heads", "kv_heads", "dim", "block"))
    blocks = lambda n: -(-n // T)  # noqa: E731
    bytes_ = flops = 0
    if case["op"] == "append":
        for n, w in zip(lens, new):
            first = (n - w) // T * T
            bytes_ += w * 2 * KH * D * 3                            # keys and values in 16 bits read, codes written
            bytes_ += (n - first) * 2 * KH * D * 3                  # codes read back, 16 bits written
            bytes_ += (blocks(n) - first // T) * 2 * KH * 4 * 2     # scales
    elif case["op"] == "attention":
        for n, w in zip(lens, new):
            bytes_ += n * 2 * KH * D + blocks(n) * 2 * KH * 4 + w * H * (4 * D + 4)
            pairs = w * (n - w) + w * (w + 1) // 2
            flops += 4 * D * H * pairs
            if case["scores"]:
                bytes_ += 8 * n * KH
    else:
        for n in lens:
            keep = min(n, case["budget"])
            bytes_ += n * KH * 4 + keep * KH * (4 + 4)              # scores read, the kept ones and their places written
            bytes_ += keep * KH * 2 * D * (2 + 3)                   # codes moved, then read back in 16 bits
            bytes_ += (min(blocks(n), keep) + 2 * blocks(keep)) * 2 * KH * 4
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits -----------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _sizes(case)
    return {"append": _exact_append, "attention": _exact_attention, "evict": _exact_evict}[case["op"]](s, case, lens, new)


def _codes64(x, scale):
    """Codes of the float64 values x under the float32 scale, as whole float64 numbers."""
    scale = scale.double()
    return torch.clamp(torch.round(x / torch.where(scale == 0, 1.0, scale)), -127, 127) * (scale != 0)


def _exact_append(s, case, lens, new):
    T = case["block"]
    value, scales = s["codes"].double(), s["scales"].clone()
    got, row = [[], []], 0
    for b, (n, w) in enumerate(zip(lens, new)):
        begin = n - w
        for j in range(begin // T, -(-n // T)):
            block = int(s["table"][b, j])
            lo, hi = max(begin, j * T), min(n, (j + 1) * T)
            for which, name in enumerate("kv"):
                x = s[name][row + lo - begin:row + hi - begin].double().transpose(0, 1)         # [kv_heads][tokens][dim]
                scale = (x.abs().amax((1, 2)) / 127).float()
                if lo > j * T:
                    scale = torch.maximum(scale, s["scales"][block, which])
                    by = torch.where(scale > 0, s["scales"][block, which].double() / scale.double(), 0.0)
                    value[block, which, :, :lo - j * T] = torch.round(value[block, which, :, :lo - j * T] * by[:, None, None])
                value[block, which, :, lo - j * T:hi - j * T] = _codes64(x, scale[:, None, None])
                scales[block, which] = scale
                got[which].append((value[block, which, :, :hi - j * T] * scale.double()[:, None, None]).transpose(0, 1))
        row += w
    return {"k": torch.cat(got[0]), "v": torch.cat(got[1]), "scales": scales.double()}


def _exact_attention(s, case, lens, new):
    H, KH, D, T = (case[k] for k in ("heads", "kv_heads", "dim", "block"))
    G, row = H // KH, 0
    out = torch.zeros((s["m"], H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((s["m"], H), float("-inf"), dtype=torch.float64, device="cuda")
    score = s["score_out"].double() if case["scores"] else None
    for b, (n, w) in enumerate(zip(lens, new)):
        at = s["table"][b, :-(-n // T)].long()
        hidden = torch.arange(n, device="cuda")[None] > torch.arange(n - w, n, device="cuda")[:, None]
        for h in range(KH):
            k, v = ((s["codes"][at, x, h].double() * s["scales"][at, x, h].double()[:, None, None]).reshape(-1, D)[:n] for x in (0, 1))
            q = s["q"][row:row + w, h * G:(h + 1) * G].double()
            logit = (torch.einsum("igd,td->igt", q, k) * s["softmax_scale"]).masked_fill_(hidden[:, None], float("-inf"))
            norm = torch.logsumexp(logit, -1)
            p = torch.exp(logit - norm[..., None])
            out[row:row + w, h * G:(h + 1) * G] = torch.einsum("igt,td->igd", p, v)
            lse[row:row + w, h * G:(h + 1) * G] = norm
            if score is not None:
                t = torch.arange(n, device="cuda")
                score[at[t // T], h, t % T] = s["score"][at[t // T], h, t % T].double() + p.sum((0, 1))
        row += w
    return {"out": out, "lse": lse, **({"score": score} if score is not None else {})}


def _exact_evict(s, case, lens, new):
    KH, D, T, budget, recent = (case[k] for k in ("kv_heads", "dim", "block", "budget", "recent"))
    scales, score = s["scales"].double(), s["score"].double()
    got = [[], []]
    kept = torch.full_like(s["kept"], -1)
    for b, n in enumerate(lens):
        count = min(n, budget)
        src, dst = s["table"][b].long(), s["dst_table"][b].long()
        t = torch.arange(n, device="cuda")
        mine = s["score"][src[t // T], :, t % T].double()                              # [tokens][kv_heads]
        if n > budget:
            # the place of a token in the order of falling score, equal ones by rising index
            old = torch.sort(-mine[:n - recent], dim=0, stable=True)[1][:budget - recent]
            keep = torch.cat([torch.sort(old, dim=0)[0], t[n - recent:, None].expand(-1, KH)])
        else:
            keep = t[:, None].expand(-1, KH)
        kept[b, :, :count] = keep.transpose(0, 1).int()
        slot = torch.arange(count, device="cuda")
        score[dst[slot // T], :, slot % T] = mine.gather(0, keep)
        for which in (0, 1):
            parts = []
            for h in range(KH):
                block = src[keep[:, h] // T]
                x = (s["codes"][block, which, h, keep[:, h] % T].float() * s["scales"][block, which, h][:, None]).double()
                whole = torch.zeros((-(-count // T) * T, D), dtype=torch.float64, device="cuda")
                whole[:count] = x
                whole = whole.view(-1, T, D)
                scale = (whole.abs().amax((1, 2)) / 127).float()
                scales[dst[:scale.shape[0]], which, h] = scale.double()
                parts.append((_codes64(whole, scale[:, None, None]) * scale.double()[:, None, None]).view(-1, D)[:count])
            got[which].append(torch.stack(parts, 1))
    return {"k": torch.cat(got[0]), "v": torch.cat(got[1]), "kept": kept, "lens": torch.tensor([min(n, budget) for n in lens], dtype=torch.int32,
            device="cuda"), "scales": scales, "score": score}
