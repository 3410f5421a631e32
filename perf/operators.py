"""Measured cases of the paged cache: what a serving program does with the keys and
values that a selection kept. The kept rows of a prompt are written into pages
(quantised to 8 bits on the way, or as they are), new tokens' rows are appended,
rows are read back, and the new tokens' queries attend to the pages.

A case names its kind:
  fill    mmshift_cache_fill: kept rows of K and V into pages;
  append  mmshift_cache_append: new tokens' rows behind them;
  read    mmshift_cache_read: rows of the pages as K and V;
  attend  mmshift_cache_attention: queries of a chunk of new tokens over the pages.
``new`` lists the new tokens of each request, ``rows`` the rows that its
sequences hold (the new ones included), ``seq`` and ``budgets`` a fill's prompt
lengths and budgets. Every (request, KV head) has its own sequence and its own
pages; with ``jitter`` the heads' lengths differ, as under budgets per head.
What an 8-bit cache was given is read back, so that it is returned as values.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}
_SIZE = {"bf16": 2, "f32": 4, "i8": 1}


def _case(name, kind, hq=28, hkv=4, d=128, dtype="bf16", cache="bf16", page=64, layers=1, new="", rows="",
          seq="", budgets="", jitter=0.0, strided=False, causal=True):
    return {"name": name, "kind": kind, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "cache": cache,
            "page": page, "layers": layers, "new": new, "rows": rows, "seq": seq, "budgets": budgets,
            "jitter": jitter, "strided": strided, "causal": causal}


def listed():
    return [
        # compaction after prefill: the 28-layer 32K stack's kept rows into an
        # 8-bit cache, and the rows as they now stand
        _case("fill_stack_32k_i8", "fill", cache="i8", layers=28, seq="32768", budgets="2048"),
        # kept rows of ragged float32 prompts with a budget for each head
        _case("fill_f32_head_budgets", "fill", hq=8, hkv=2, d=64, dtype="f32", cache="f32", page=16, layers=3,
              seq="4001,700,33", budgets="640,129,33", jitter=0.5),
        # one decode step of one request: the smallest call
        _case("append_token", "append", new="1", rows="1025"),
        # the prompts' next turns, ragged, rows inside a fused projection's output,
        # into an 8-bit cache, and what it holds of them
        _case("append_chunks_i8", "append", hq=64, hkv=8, cache="i8", page=128, new="512,1,77,1024,300,8,200,64",
              rows="2560,193,4096,1100,9000,300,200,777", strided=True),
        # a 72B-class layer's sequences read back as bfloat16 rows (to move or to re-score them)
        _case("read_72b_i8", "read", hq=64, hkv=8, cache="i8", page=64, rows="2048,24576,4096,6000,8192,12000,16384,3001"),
        # odd float32 rows, small pages
        _case("read_f32_odd", "read", hq=8, hkv=2, d=64, dtype="f32", cache="f32", page=16, rows="1,1500,37", jitter=0.4),
        # one decode step over one compacted cache: latency
        _case("attend_token_1k", "attend", new="1", rows="1025"),
        # a decode step of a full batch, long 8-bit caches, lengths that differ by head: bandwidth
        _case("attend_batch_i8", "attend", hq=64, hkv=8, cache="i8", page=64, new=",".join(["1"] * 64),
              rows=",".join(str(2048 + 347 * (i * 37 % 64)) for i in range(64)), jitter=0.2),
        # verification of eight drafted tokens, heads of their own (no grouping), small pages
        _case("attend_drafts", "attend", hq=32, hkv=32, page=16, new=",".join(["8"] * 16),
              rows=",".join(str(700 + 101 * i) for i in range(16))),
        # the next chunk of a long prompt over an uncompacted cache: the largest, matrix products
        _case("attend_chunk_2k_over_32k", "attend", page=128, new="2048", rows="34816"),
        # ragged turns of a mixed batch over 8-bit compacted caches
        _case("attend_turns_i8", "attend", cache="i8", page=32, new="1024,1,300,17,513", rows="3100,2049,8000,17,1025",
              jitter=0.1),
        # float32, odd chunk and length
        _case("attend_f32_chunk", "attend", hq=8, hkv=2, d=64, dtype="f32", cache="f32", page=16, new="257", rows="4001"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend"] * 5 + ["fill", "append", "read"])
    hq, hkv, d = rng.choice([(28, 4, 128), (64, 8, 128), (8, 2, 64), (32, 8, 128), (4, 1, 64), (32, 32, 128), (16, 16, 64)])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    cache = "i8" if rng.random() < 0.45 else dtype
    page = rng.choice([16, 32, 64, 128, 256])
    batch = rng.choice([1, 1, 2, 3, 5, 8, 16, 33, 64])
    jitter = rng.choice([0.0, 0.0, 0.15, 0.5])
    c = dict(hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, page=page, jitter=jitter)
    if kind == "fill":
        batch = min(batch, 8)
        seq = [_log_int(rng, 40, 32768 // batch) for _ in range(batch)]
        frac = math.exp(rng.uniform(math.log(0.02), math.log(0.6)))
        budgets = [max(1, round(frac * t)) for t in seq]
        return _case("", kind, **c, layers=rng.choice([1, 2, 7, 28]) if hkv * d <= 1024 else 2,
                     seq=_text(seq), budgets=_text(budgets))
    # at most 1.5 million rows of all heads, as the listed batch has
    rows = [_log_int(rng, 1, min(32768, 1500000 // (hkv * batch))) for _ in range(batch)]
    if kind == "read":
        return _case("", kind, **c, rows=_text(rows))
    shape = rng.choice(["tokens", "drafts", "chunks", "mixed"])
    most = {"tokens": 1, "drafts": 16, "chunks": 2048, "mixed": 1024}[shape]
    new = [1 if most == 1 or (shape == "mixed" and rng.random() < 0.5) else _log_int(rng, 2, most) for _ in rows]
    rows = [max(a, b) for a, b in zip(rows, new)]
    # no more products than the listed chunk has: float32's on the CUDA cores a twentieth
    limit = 28 * 2048 * 33000 / (20 if dtype == "f32" else 1)
    # (and twice its padded logits in the plain form)
    while (sum(hq * n * t for n, t in zip(new, rows)) > limit
           or hq * batch * max(new) * max(rows) > 2 * 28 * 2048 * 34816):
        new = [max(1, n // 2) for n in new]
        rows = [max(n, t * 3 // 4) for n, t in zip(new, rows)]
    return _case("", kind, **c, new=_text(new), rows=_text(rows), strided=rng.random() < 0.4,
                 causal=kind != "attend" or rng.random() < 0.85)


def _text(v):
    return ",".join(map(str, v))


def _ints(text):
    return [int(x) for x in text.split(",")]


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _new(case):
    return _ints(case["new"]) if case["new"] else [0] * len(_ints(case["rows"] or case["seq"]))


def _lens(case):
    """Rows of each (layer, request, KV head): nested lists [layers][batch][hkv]."""
    r = random.Random(20260722)
    if case["kind"] == "fill":
        full = [min(c, t) for c, t in zip(_ints(case["budgets"]), _ints(case["seq"]))]
    else:
        full = _ints(case["rows"])
    least = [max(1, n) for n in _new(case)]
    return [[[max(m, min(t, t - int(case["jitter"] * r.random() * t))) for _ in range(case["hkv"])]
             for t, m in zip(full, least)] for _ in range(case["layers"])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, ct, d, hkv, hq, L = _DT[case["dtype"]], _DT[case["cache"]], case["d"], case["hkv"], case["hq"], case["layers"]

    def randn(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    lens = torch.tensor(_lens(case), dtype=torch.int32)
    batch, page = lens.shape[1], case["page"]
    need = (lens + page - 1) // page
    most = int(need.max())
    total = int(need.sum())
    # every sequence's pages lie where the pool had room: in no order
    order = torch.randperm(total + 3, generator=gen, device="cuda")[:total].to(torch.int32)
    table = torch.full((L * batch * hkv, most), -1, dtype=torch.int32, device="cuda")
    used = torch.arange(most, device="cuda")[None] < need.reshape(-1, 1).cuda()
    table[used] = order
    s = {"case": case, "table": table.view(L, batch, hkv, most), "lens": lens.cuda(), "lmax": int(lens.max())}
    pool = (total + 3, page, d)
    if case["kind"] in ("fill", "append"):
        s["kp"], s["vp"] = torch.zeros(pool, dtype=ct, device="cuda"), torch.zeros(pool, dtype=ct, device="cuda")
        if ct == torch.int8:
            s["ks"], s["vs"] = (torch.zeros(pool[:2], device="cuda") for _ in range(2))
    elif ct == torch.int8:
        s["kp"], s["vp"] = (torch.randint(-127, 128, pool, generator=gen, device="cuda", dtype=torch.int8) for _ in range(2))
        # a row of 128 normal values has its largest at about 2.7
        s["ks"], s["vs"] = (torch.rand(pool[:2], generator=gen, device="cuda") * 0.01 + 0.017 for _ in range(2))
    else:
        s["kp"], s["vp"] = randn(*pool, dtype=ct), randn(*pool, dtype=ct)
    if case["kind"] == "fill":
        seq, budgets = _ints(case["seq"]), _ints(case["budgets"])
        cu = _cu(seq)
        s["K"], s["V"] = randn(L, cu[-1], hkv, d), randn(L, cu[-1], hkv, d)
        parts = []
        for t, c in zip(seq, budgets):
            score = torch.rand((L, t, hkv), generator=gen, device="cuda")
            score[:, -1] = 2.0                         # the last token always stays
            parts.append(score.topk(min(c, t), dim=1).indices.sort(dim=1).values)
        idx = torch.cat(parts, dim=1).to(torch.int32)  # [L, R, hkv]
        cuk = _cu([p.shape[1] for p in parts])
        s["row_of"] = torch.cat([torch.arange(p.shape[1], device="cuda") for p in parts])
        s["req_of"] = torch.cat([torch.full((p.shape[1],), b, device="cuda") for b, p in enumerate(parts)])
        behind = s["row_of"][None, :, None] >= s["lens"][:, s["req_of"]]
        s["idx"] = idx.masked_fill(behind, -1)
        s["seq_start"] = torch.tensor(cu, device="cuda")
        s["count"] = s["lens"].clone() if case["jitter"] else None
        s["cu_out"] = cuk
    elif case["kind"] == "read":
        s["cu_out"] = _cu(_ints(case["rows"]))
    else:
        new = _new(case)
        s["cu_out"] = _cu(new)
        t = s["cu_out"][-1]
        if case["strided"]:                            # one projection's output holds q, k and v side by side
            qkv = randn(L, t, (hq + 2 * hkv) * d)
            q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=-1)
            s["stride"] = qkv.stride(1)
        else:
            q, k, v = randn(L, t, hq * d), randn(L, t, hkv * d), randn(L, t, hkv * d)
            s["stride"] = 0
        s["K"], s["V"] = k.unflatten(-1, (hkv, d)), v.unflatten(-1, (hkv, d))
        s["Q"] = q.unflatten(-1, (hq, d))[0]
        s["first"] = s["lens"] - torch.tensor(new, dtype=torch.int32, device="cuda")[None, :, None]
    if case["kind"] != "fill":
        counts = [b - a for a, b in zip(s["cu_out"], s["cu_out"][1:])]
        s["row_of"] = torch.cat([torch.arange(n, device="cuda") for n in counts])
        s["req_of"] = torch.repeat_interleave(torch.arange(batch, device="cuda"), torch.tensor(counts, device="cuda"))
        s["new"] = torch.tensor(counts, device="cuda")
        s["nmax"] = max(counts)
    rows = s["cu_out"][-1]
    if case["kind"] == "attend":
        s["out"] = torch.empty((rows, hq, d), dtype=dt, device="cuda")
        s["lse"] = torch.empty((rows, hq), device="cuda")
    elif case["kind"] == "read" or ct == torch.int8:
        s["out_k"] = torch.empty((L, rows, hkv, d), dtype=dt, device="cuda")
        s["out_v"] = torch.empty_like(s["out_k"])
    if own:
        _handles(s, case)
    return s


def _handles(s, case):
    """The shape, cache and workspace that a serving program keeps for a call."""
    import paper_2607_22586_gb300 as M

    dt = 0 if case["dtype"] == "bf16" else 1
    L = case["layers"]
    cache = M.make_cache(s["kp"], s["vp"], s["table"], s["lens"], s.get("ks"), s.get("vs"))

    def shape(cu, budgets, stride_kv):
        return M.make_shape(case["hq"], case["hkv"], case["d"], 2, dt, cu, budgets, n_layers=L,
                            layer_stride_kv=stride_kv, layer_stride_q=len(budgets) * 2 * case["hq"] * case["d"])

    rows = shape(s["cu_out"], [1] * (len(s["cu_out"]) - 1), s["K"].stride(0) if "K" in s else 0)
    n = M.mmshift_cache_workspace_size(rows, cache)
    s["own"] = {"M": M, "cache": cache, "rows": rows, "n": n, "ws": torch.zeros(n, dtype=torch.uint8, device="cuda")}
    if case["kind"] == "fill":
        seq = _ints(case["seq"])
        s["own"]["prompt"] = shape(_cu(seq), _ints(case["budgets"]), s["K"].stride(0))


def run(s):
    case = s["case"]
    kind, quantised = case["kind"], case["cache"] == "i8"
    if own:
        o = s["own"]
        M, rest = o["M"], (o["ws"], o["n"], torch.cuda.current_stream())
        if kind == "attend":
            M.check(M.mmshift_cache_attention(o["rows"], o["cache"], s["Q"], s["stride"], case["causal"], 0.0,
                                              s["out"], s["lse"], *rest), "attention")
            return {"out": s["out"], "lse": s["lse"]}
        if kind == "fill":
            M.check(M.mmshift_cache_fill(o["prompt"], o["cache"], s["K"], s["V"], s["idx"], s["count"], *rest), "fill")
        elif kind == "append":
            M.check(M.mmshift_cache_append(o["rows"], o["cache"], s["K"], s["V"], s["stride"], *rest), "append")
        if kind == "read" or quantised:
            first = s["first"] if kind == "append" else None
            M.check(M.mmshift_cache_read(o["rows"], o["cache"], first, s["out_k"], s["out_v"], *rest), "read")
            got = {"k": s["out_k"], "v": s["out_v"]}
        else:
            got = {"k": s["kp"], "v": s["vp"]}
        return {**got, "lens": s["lens"]} if kind == "fill" else got
    if kind == "attend":
        return _attend(s, case)
    if kind == "fill":
        token = s["seq_start"][s["req_of"]][None, :, None] + s["idx"].clamp(min=0)
        k, v = (x.gather(1, token[..., None].expand(-1, -1, -1, case["d"])) for x in (s["K"], s["V"]))
        pos, there = s["row_of"][None, :, None].expand(token.shape), s["idx"] >= 0
    elif kind == "append":
        k, v = s["K"], s["V"]
        pos = s["row_of"][None, :, None] + s["first"][:, s["req_of"]]
        there = pos >= 0
    if kind == "read":
        pos = s["row_of"][None, :, None].expand(case["layers"], -1, case["hkv"])
        there = pos < s["lens"][:, s["req_of"]]
    # the pool's row of each position: [layers, rows, hkv]
    entry = s["table"][:, s["req_of"]].gather(-1, (pos // case["page"]).clamp(0, s["table"].shape[-1] - 1).long()[..., None])
    slot = entry[..., 0].long() * case["page"] + pos % case["page"]
    if kind != "read":
        for x, pages, scales in ((k, s["kp"], s.get("ks")), (v, s["vp"], s.get("vs"))):
            if quantised:
                code, scale = _quantise(x)
                pages.view(-1, case["d"])[slot[there]] = code[there]
                scales.view(-1)[slot[there]] = scale[there]
            else:
                pages.view(-1, case["d"])[slot[there]] = x[there]
    if kind != "read" and not quantised:
        got = {"k": s["kp"], "v": s["vp"]}
    else:
        slot = slot.masked_fill(~there, 0)
        got = {n: _values(s, n, slot).masked_fill(~there[..., None], 0).to(_DT[case["dtype"]]) for n in "kv"}
    return {**got, "lens": s["lens"]} if kind == "fill" else got


def _quantise(x):
    """A row's codes in [-127, 127] and its scale: its largest magnitude over 127.
    Both quotients are of two tensors: by or of a number, torch multiplies by a reciprocal."""
    x = x.float()
    most = x.abs().amax(-1, keepdim=True)
    full = torch.full_like(most, 127.0)
    code = torch.round(x * (full / most.clamp(min=2.0 ** -110))).to(torch.int8)
    return code, (most / full)[..., 0]


def _values(s, name, slot):
    x = s[name + "p"].view(-1, s["case"]["d"])[slot].float()
    return x * s[name + "s"].view(-1)[slot][..., None] if s["case"]["cache"] == "i8" else x


def _attend(s, case):
    hkv, r, d, dev = case["hkv"], case["hq"] // case["hkv"], case["d"], s["Q"].device
    batch, nmax = len(s["new"]), s["nmax"]
    pos = torch.arange(s["lmax"], device=dev)
    lens = s["lens"][0]                                                # [batch, hkv]
    slot = s["table"][0].long()[..., pos // case["page"]] * case["page"] + pos % case["page"]
    slot = slot.masked_fill(pos >= lens[..., None], 0)
    q = torch.zeros((batch, nmax, case["hq"], d), device=dev)
    q[s["req_of"], s["row_of"]] = s["Q"].float()
    q = q.unflatten(2, (hkv, r)).permute(0, 2, 1, 3, 4).reshape(batch, hkv, nmax * r, d)
    logits = (q @ _values(s, "k", slot).transpose(-1, -2)).view(batch, hkv, nmax, r, -1) * d ** -0.5
    limit = lens[..., None].expand(-1, -1, nmax)
    if case["causal"]:
        limit = limit - s["new"][:, None, None] + torch.arange(1, nmax + 1, device=dev)
    logits.masked_fill_(pos >= limit[..., None, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    e = logits.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    v = _values(s, "v", slot).masked_fill((pos >= lens[..., None])[..., None], 0)
    out = (e.flatten(2, 3) @ v).view(batch, hkv, nmax, r, d) / total.clamp(min=1e-38)
    lse = (top + total.log())[..., 0]
    back = lambda x: x.transpose(1, 2).flatten(2, 3)[s["req_of"], s["row_of"]]  # noqa: E731
    return {"out": back(out).to(_DT[case["dtype"]]), "lse": back(lse)}


def work(case):
    d, hkv, hq, esz, csz = case["d"], case["hkv"], case["hq"], _SIZE[case["dtype"]], _SIZE[case["cache"]]
    lens, new = _lens(case), _new(case)
    row = d * csz + (4 if case["cache"] == "i8" else 0)                # a row in the pages
    held = sum(t for layer in lens for unit in layer for t in unit)
    if case["kind"] == "attend":
        t = sum(new)
        pairs = 0
        for unit, n in zip(lens[0], new):
            for m in unit:
                first = m - n + 1 if case["causal"] else m             # keys of the chunk's first token
                pairs += n * first + (n * (n - 1) // 2 if case["causal"] else 0)
        kv = 2 * row * sum(m for unit, n in zip(lens[0], new) if n for m in unit)
        return {"bytes": kv + 2 * t * hq * d * esz + 4 * t * hq, "flops": 4.0 * d * (hq // hkv) * pairs}
    if case["kind"] == "append":
        held = sum(new) * hkv * case["layers"]
    rows = held
    if case["kind"] == "read":
        rows = sum(_ints(case["rows"])) * hkv
        return {"bytes": 2 * (held * row + rows * d * esz), "flops": 0}
    bytes_ = 2 * held * (d * esz + row) + (4 * held if case["kind"] == "fill" else 0)
    if case["cache"] == "i8":                                          # read back
        if case["kind"] == "fill":
            rows = sum(min(c, t) for c, t in zip(_ints(case["budgets"]), _ints(case["seq"]))) * hkv * case["layers"]
        bytes_ += 2 * (held * row + rows * d * esz)
    return {"bytes": bytes_, "flops": 0}


def exact(case, seed):
    """Attention and 8-bit rows from their formulas in float64, one sequence at a time;
    copies of rows are no computed numbers."""
    if case["kind"] != "attend" and case["cache"] != "i8":
        return None
    s = prepare(case, seed)
    hkv, hq, d, page = case["hkv"], case["hq"], case["d"], case["page"]
    r, lens, cu, new = hq // hkv, _lens(case), s["cu_out"], _new(case)

    def sequence(l, b, h, name):
        rows = s[name + "p"][s["table"][l, b, h, :(lens[l][b][h] + page - 1) // page].long()].double()
        if case["cache"] == "i8":
            rows = rows * s[name + "s"][s["table"][l, b, h, :rows.shape[0]].long()].double()[..., None]
        return rows.reshape(-1, d)[:lens[l][b][h]]

    if case["kind"] == "attend":
        out = torch.zeros((cu[-1], hq, d), dtype=torch.float64, device="cuda")
        lse = torch.zeros((cu[-1], hq), dtype=torch.float64, device="cuda")
        for b, n in enumerate(new):
            for h in range(hkv):
                k, v, m = sequence(0, b, h, "k"), sequence(0, b, h, "v"), lens[0][b][h]
                seen = torch.arange(m, device="cuda")[None] < torch.arange(m - n + 1, m + 1, device="cuda")[:, None]
                for j in range(h * r, (h + 1) * r):
                    z = s["Q"][cu[b]:cu[b + 1], j].double() @ k.T / math.sqrt(d)
                    if case["causal"]:
                        z = torch.where(seen, z, -math.inf)
                    lse[cu[b]:cu[b + 1], j] = torch.logsumexp(z, -1)
                    out[cu[b]:cu[b + 1], j] = torch.softmax(z, -1) @ v
        return {"out": out, "lse": lse}
    got = {n: torch.zeros(s["out_k"].shape, dtype=torch.float64, device="cuda") for n in "kv"}
    for l in range(case["layers"]):
        for b in range(len(lens[l])):
            for h in range(hkv):
                m, at = lens[l][b][h], cu[b]
                for n in "kv":
                    if case["kind"] == "read":
                        got[n][l, at:at + m, h] = sequence(l, b, h, n)
                        continue
                    if case["kind"] == "fill":
                        start = _cu(_ints(case["seq"]))[b]
                        x = s[n.upper()][l, start + s["idx"][l, at:at + m, h].long(), h].double()
                    else:
                        m = new[b]
                        x = s[n.upper()][l, at:at + m, h].double()
                    step = x.abs().amax(-1, keepdim=True) / 127
                    got[n][l, at:at + m, h] = torch.round(x / step) * step
    return {**got, "lens": None} if case["kind"] == "fill" else got
