"""Measured cases of what a serving program does around a selection and its paged cache:
Q and K of new tokens are rotated to their positions, a prompt's tokens attend to one
another, a prompt's pages are shared by several answers, trimmed and given back, and
the answers' tokens attend to pages that they share.

A case names its kind:
  rope     mmshift_rope: rotary positions of Q and K rows;
  prompt   mmshift_prompt_attention: attention over whole packed prompts;
  fork     mmshift_cache_fork, _reserve and _append: sequences that share a prompt's
           pages, and the first new tokens of each;
  branch   mmshift_cache_fork and _compact: a copy of a sequence that keeps some rows;
  refill   mmshift_cache_free, _reserve, _fill and _compact: a prompt's rows into pages
           that were free, then some of them kept, in place;
  shared   mmshift_cache_attention_shared: new tokens' queries over sequences that share
           pages.
``new`` lists the new tokens of each request (rope, prompt: its tokens), ``rows`` the
rows that its sequences hold (shared: the new ones included). fork and branch: the first
len(rows) requests hold prompts, each of which ``answers`` further requests take over.
shared: ``answers`` requests in a row share ``prefix`` rows' pages (a number for each
group). ``keep``: rows kept by a compaction. Every (request, KV head) has its own
sequence; with ``jitter`` the heads' lengths differ. What an 8-bit cache holds is read
back, so that it is returned as values.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32, "i8": torch.int8}
_SIZE = {"bf16": 2, "f32": 4, "i8": 1}


def _case(name, kind, hq=28, hkv=4, d=128, dtype="bf16", cache="bf16", page=64, layers=1, new="", rows="", answers=1,
          prefix="", keep="", jitter=0.0, strided=False, causal=True, layout="half", rot=0, sections="", scaling="none",
          factor=1.0, far=0):
    return {"name": name, "kind": kind, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "cache": cache, "page": page,
            "layers": layers, "new": new, "rows": rows, "answers": answers, "prefix": prefix, "keep": keep,
            "jitter": jitter, "strided": strided, "causal": causal, "layout": layout, "rot": rot,
            "sections": sections, "scaling": scaling, "factor": factor, "far": far}


def listed():
    return [
        # a decode step of a batch, far into long answers: latency
        _case("rope_tokens_far", "rope", hq=32, hkv=8, new=",".join(["1"] * 16), layout="interleaved", rot=64,
              scaling="parts", factor=16.0, far=1000000),
        # a prompt of text and images with three position axes, out of a fused projection's rows: bandwidth
        _case("rope_prompt_32k", "rope", new="32768", strided=True, sections="16,24,24"),
        # a batch of ragged prompts, short ones among them
        _case("prompt_ragged", "prompt", new="17,1000,301,1500,64,777,129,1024,5,640,1,2048,350,900,1100,513", strided=True),
        # a long prompt: the largest, matrix products
        _case("prompt_32k", "prompt", new="32768"),
        # images' patches, which see all of their image, heads of their own
        _case("prompt_images", "prompt", hq=16, hkv=16, d=64, new="1036,529,2116,37", causal=False),
        # float32, odd lengths
        _case("prompt_f32", "prompt", hq=8, hkv=2, d=64, dtype="f32", new="1501,33,700"),
        # eight answers to a compacted prompt: its pages shared by 28 layers, the first tokens' rows
        _case("fork_answers", "fork", layers=28, rows="2072", answers=8, new="1"),
        # drafted tokens of many answers to ragged prompts, heads of their own lengths, 8-bit rows
        _case("fork_ragged_i8", "fork", hq=64, hkv=8, cache="i8", page=32, layers=8, rows="1300,77,4000,513", answers=12,
              new="5", jitter=0.3),
        # a branch that keeps half of its rows, next to the sequence that keeps all
        _case("branch_half", "branch", layers=28, rows="4100", keep="2048"),
        # the rows of float32 prompts into free pages, then fewer of them, where they are
        _case("refill_f32", "refill", hq=8, hkv=2, d=64, dtype="f32", cache="f32", page=16, layers=3, rows="4001,700,33",
              keep="1900,256,33"),
        # a decode step of 64 answers to one long prompt: the prompt read once
        _case("shared_answers", "shared", hq=64, hkv=8, new=",".join(["1"] * 64), prefix="24000", answers=64,
              rows=",".join(str(24100 + 37 * (i * 37 % 64)) for i in range(64))),
        # verification of drafts of groups of answers to ragged prompts, 8-bit pages, heads of their own lengths
        _case("shared_drafts_i8", "shared", cache="i8", page=32, answers=4, prefix="8000,517,3000", jitter=0.1,
              new="4,4,1,4,6,6,6,6,1,8,1,2", rows="8333,8100,8004,9000,700,523,611,900,3001,3500,4444,3100"),
    ]


_HEADS = [(28, 4, 128), (64, 8, 128), (8, 2, 64), (32, 8, 128), (4, 1, 64), (32, 32, 128), (16, 16, 64), (20, 4, 128)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "prompt", "prompt", "fork", "branch", "refill", "shared", "shared"])
    hq, hkv, d = rng.choice(_HEADS)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    cache = "i8" if kind not in ("rope", "prompt") and rng.random() < 0.4 else dtype
    c = dict(hq=hq, hkv=hkv, d=d, dtype=dtype, cache=cache, page=rng.choice([16, 32, 64, 128, 256]))
    strided = rng.random() < 0.4
    if kind == "rope":
        batch = rng.choice([1, 1, 3, 8, 64])
        new = [_log_int(rng, 1, 32768 // batch // max(hkv // 4, 1)) for _ in range(batch)]
        rot = rng.choice([0, d // 2, d // 4 * 3, 24])
        scaling = rng.choice(["none", "linear", "base", "parts"])
        n = (rot or d) // 2
        a = n // 4
        return _case("", kind, **c, new=_text(new), strided=strided, layout=rng.choice(["half", "interleaved"]), rot=rot,
                     sections="" if rng.random() < 0.6 else _text([a, (n - a) // 2, n - a - (n - a) // 2]),
                     scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 16.0, 40.0]),
                     far=rng.choice([0, 0, 100000, 4000000]))
    if kind == "prompt":
        batch = rng.choice([1, 1, 2, 5, 16, 64])
        new = [_log_int(rng, 1, 32768 // batch) for _ in range(batch)]
        causal = rng.random() < 0.75
        # no more products than the listed prompt has: float32's on the CUDA cores a twentieth
        limit = 28 * 32768 ** 2 * 128 / (20 if dtype == "f32" else 1) / (1 if causal else 2)
        while sum(hq * n * n * d for n in new) > limit:
            new = [max(1, n * 3 // 4) for n in new]
        return _case("", kind, **c, new=_text(new), strided=strided, causal=causal)
    jitter = rng.choice([0.0, 0.0, 0.15, 0.5])
    layers = rng.choice([1, 2, 7, 28]) if hkv * d <= 1024 else rng.choice([1, 2])
    if kind in ("fork", "branch"):
        prompts = rng.choice([1, 1, 2, 4])
        answers = 1 if kind == "branch" else _log_int(rng, 1, 60 // prompts)
        rows = [_log_int(rng, 1, 8192 // prompts) for _ in range(prompts)]
        if kind == "fork":
            return _case("", kind, **c, layers=layers, rows=_text(rows), answers=answers, jitter=jitter,
                         new=str(rng.choice([1, 1, 3, 8, 65, 300])), strided=strided)
        return _case("", kind, **c, layers=layers, rows=_text(rows), jitter=jitter,
                     keep=_text([max(1, int(n * rng.uniform(0.1, 1.0))) for n in rows]))
    if kind == "refill":
        batch = rng.choice([1, 2, 3, 8])
        rows = [_log_int(rng, 1, 8192 // batch) for _ in range(batch)]
        return _case("", kind, **c, layers=layers, rows=_text(rows),
                     keep=_text([max(1, int(n * rng.uniform(0.1, 1.0))) for n in rows]))
    groups = rng.choice([1, 1, 2, 5])
    answers = _log_int(rng, 2, 64 // groups)
    prefix = [_log_int(rng, 1, min(32768, 2000000 // (hkv * groups))) for _ in range(groups)]
    most = rng.choice([1, 1, 8, 40, 300]) if dtype == "bf16" else rng.choice([1, 8])
    new, rows = [], []
    for p in prefix:
        for _ in range(answers):
            new.append(1 if most == 1 else _log_int(rng, 1, most))
            rows.append(p + new[-1] + _log_int(rng, 1, min(3000, 400000 // (hkv * answers * groups))) - 1)
    while sum(hq * n * t for n, t in zip(new, rows)) > 28 * 2048 * 33000 / (20 if dtype == "f32" else 1):
        new = [max(1, n // 2) for n in new]
        if max(new) == 1:
            prefix = [max(1, p * 3 // 4) for p in prefix]
            rows = [p + 5 for p in prefix for _ in range(answers)]
    return _case("", kind, **c, new=_text(new), rows=_text(rows), prefix=_text(prefix), answers=answers, jitter=jitter,
                 strided=strided, causal=rng.random() < 0.85)


def _text(v):
    return ",".join(map(str, v))


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _new(case):
    """New tokens of each request."""
    if case["kind"] == "fork":
        prompts = len(_ints(case["rows"]))
        return [0] * prompts + _ints(case["new"]) * (prompts * case["answers"])
    if case["kind"] == "branch":
        return [0] * len(_ints(case["rows"])) + _ints(case["keep"])
    return _ints(case["keep"] if case["kind"] == "refill" else case["new"])


def _frequencies(case):
    """Radians a position of each pair, and what the rotated values are multiplied by."""
    n, theta, s, original = (case["rot"] or case["d"]) // 2, 1e6, case["factor"], 32768
    if case["scaling"] == "base":
        theta *= s ** (n / (n - 1))
    f = [theta ** (-j / n) for j in range(n)]
    if case["scaling"] == "linear":
        f = [x / s for x in f]
    if case["scaling"] != "parts":
        return f, 1.0
    # frequencies of many turns within the original length stay, those of few are divided
    ramp = [min(max((original * x / (2 * math.pi) - 1) / (32 - 1), 0.0), 1.0) for x in f]
    return [x * r + x / s * (1 - r) for x, r in zip(f, ramp)], 0.1 * math.log(s) + 1


def _lens(case):
    """Rows of each (layer, request, KV head) that the requests of ``rows`` hold, and of
    shared the rows that a group's sequences have in common: nested lists."""
    r = random.Random(20260722)
    rows = _ints(case["rows"])

    def some(t, least=1):
        return [max(least, t - int(case["jitter"] * r.random() * t)) for _ in range(case["hkv"])]

    if case["kind"] != "shared":
        return [[some(t) for t in rows] for _ in range(case["layers"])], None
    common = [some(p) for p in _ints(case["prefix"])]
    new = _new(case)
    g = [b // case["answers"] for b in range(len(rows))]
    own_rows = [t - _ints(case["prefix"])[g[b]] for b, t in enumerate(rows)]
    return [[[p + max(n, m - int(case["jitter"] * r.random() * m)) for p in common[g[b]]]
             for b, (m, n) in enumerate(zip(own_rows, new))]], common


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, ct, d, hkv, hq, L = _DT[case["dtype"]], _DT[case["cache"]], case["d"], case["hkv"], case["hq"], case["layers"]
    kind, page, new = case["kind"], case["page"], _new(case)
    s = {"case": case}

    def randn(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    cu = s["cu"] = _cu(new)
    total = cu[-1]
    if case["strided"]:                                # one projection's output holds q, k and v side by side
        q, k, v = randn(L, total, (hq + 2 * hkv) * d).split([hq * d, hkv * d, hkv * d], dim=-1)
    elif kind not in ("branch", "refill"):
        q, k, v = randn(L, total, hq * d), randn(L, total, hkv * d), randn(L, total, hkv * d)
    if kind not in ("branch", "refill"):
        s["Q"], s["K"], s["V"] = q.unflatten(-1, (hq, d))[0], k.unflatten(-1, (hkv, d)), v.unflatten(-1, (hkv, d))
        s["out"] = torch.empty((total, hq, d), dtype=dt, device="cuda")
    if kind == "rope":
        # consecutive tokens of a request, behind what its cache holds; images' rows and columns differ from time
        first = torch.randint(0, case["far"] + 1, (len(new),), generator=gen, device="cuda")
        at = torch.cat([torch.arange(n, device="cuda") + first[b] for b, n in enumerate(new)])
        axes = [at] + [at + torch.randint(0, 48, (total,), generator=gen, device="cuda")
                       for _ in _ints(case["sections"])[1:]]
        s["positions"] = torch.stack(axes).to(torch.int32)
        s["out_k"] = torch.empty((total, hkv, d), dtype=dt, device="cuda")
        f, s["amplitude"] = _frequencies(case)
        s["freq"] = torch.tensor(f, dtype=torch.float64, device="cuda")
        of = _ints(case["sections"]) or [len(f)]
        s["axis"] = torch.repeat_interleave(torch.arange(len(of), device="cuda"), torch.tensor(of, device="cuda"))
    elif kind in ("prompt", "shared"):
        s["lse"] = torch.empty((total, hq), device="cuda")
    if kind in ("fork", "branch", "refill", "shared"):
        _pages(s, case, gen, randn, ints)
    if own:
        _handles(s, case)
    return s


def _pages(s, case, gen, randn, ints):
    """The pool, the table, the lengths and the number of sequences that hold each page."""
    kind, page, L, hkv, d, ct = case["kind"], case["page"], case["layers"], case["hkv"], case["d"], _DT[case["cache"]]
    rows, new = _ints(case["rows"]), _new(case)
    held, common = _lens(case)
    B = len(new)
    lens = torch.zeros((L, B, hkv), dtype=torch.int32)
    lens[:, :len(rows)] = torch.tensor(held, dtype=torch.int32)
    if kind == "refill":                               # what the prompts' fill leaves
        s["full"], s["keep"] = lens.cuda(), ints(_ints(case["keep"]))
    room = lens.clone()                                # rows that there have to be pages for
    for b in range(len(rows), B):
        room[:, b] = lens[:, (b - len(rows)) // case["answers"]] + (new[b] if kind == "fork" else 0)
    need = (room + page - 1) // page
    most, pool = int(need.max()), int(need.sum()) + 7
    have = (lens + page - 1) // page
    total = int(have.sum())
    # every sequence's pages lie where the pool had room: in no order
    order = torch.randperm(pool, generator=gen, device="cuda")[:total].to(torch.int32)
    table = torch.full((L * B * hkv, most), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(most, device="cuda")[None] < have.reshape(-1, 1).cuda()] = order
    table = table.view(L, B, hkv, most)
    if kind == "shared":                               # whole pages of the common rows are the first request's
        for b in range(B):
            b0 = b // case["answers"] * case["answers"]
            full = ints([p // page for p in common[b // case["answers"]]])
            same = torch.arange(most, device="cuda")[None] < full[:, None]
            table[0, b] = torch.where(same, table[0, b0], table[0, b])
    refs = torch.zeros(pool, dtype=torch.int32, device="cuda")
    refs.index_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    s["table"], s["lens"], s["refs"] = table, lens.cuda(), refs
    shape = (pool, page, d)
    if ct == torch.int8:
        s["kp"], s["vp"] = (torch.randint(-127, 128, shape, generator=gen, device="cuda", dtype=torch.int8) for _ in range(2))
        # a row of 128 normal values has its largest at about 2.7
        s["ks"], s["vs"] = (torch.rand(shape[:2], generator=gen, device="cuda") * 0.01 + 0.017 for _ in range(2))
    else:
        s["kp"], s["vp"] = randn(*shape, dtype=ct), randn(*shape, dtype=ct)
    if kind == "refill":
        s["table"].fill_(-1)
        s["refs"].zero_()
        seq = [2 * n for n in rows]                    # half of each prompt was selected
        s["seq"], s["cu_seq"], s["cu_fill"] = seq, _cu(seq), _cu(rows)
        s["K"], s["V"] = randn(L, s["cu_seq"][-1], hkv, d), randn(L, s["cu_seq"][-1], hkv, d)
        s["idx"] = torch.cat([_subset(gen, L, t, hkv, [[[n] * hkv]] * L, n) for t, n in zip(seq, rows)], 1)
    if kind in ("branch", "refill"):
        parts = []
        for b, n in enumerate(_ints(case["keep"])):
            src = [[held[l][b]] for l in range(L)]
            parts.append(_subset(gen, L, max(max(x[0]) for x in src), hkv, src, n, within=True))
        s["sel"] = torch.cat(parts, 1)
        # heads that hold fewer rows than are kept keep all
        kept = torch.zeros((L, B, hkv), dtype=torch.int32)
        for b, n in enumerate(_ints(case["keep"])):
            at = b + (len(rows) if kind == "branch" else 0)
            kept[:, at] = torch.tensor([held[l][b] for l in range(L)], dtype=torch.int32).clamp(max=n)
        s["kept"] = kept.cuda()
    s["new"] = ints(new)
    s["add"] = s["new"][None, :, None].expand(L, B, hkv).contiguous()
    counts = torch.tensor(new, device="cuda")
    s["req_of"] = torch.repeat_interleave(torch.arange(B, device="cuda"), counts)
    s["row_of"] = torch.cat([torch.arange(n, device="cuda") for n in new])
    if kind in ("fork", "branch"):
        s["dst"] = list(range(len(rows), B))
        s["src"] = [(b - len(rows)) // case["answers"] for b in s["dst"]]
    if ct == torch.int8 and kind != "shared":          # rows that are read back
        n = s["back"] = [0 if kind == "fork" and b < len(rows) else page + m if kind == "fork" else m
                         for b, m in enumerate(new)]
        s["cu_back"] = _cu(n)
        s["first"] = torch.zeros_like(s["lens"])
        if kind == "fork":                             # what was copied, and what is new
            after = s["lens"].clone()
            after[:, s["dst"]] = after[:, s["src"]] + s["add"][:, s["dst"]]
            s["first"] = (after - torch.tensor(n, dtype=torch.int32, device="cuda")[None, :, None]).clamp(min=0)
        s["back_req"] = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(n, device="cuda"))
        s["back_row"] = torch.cat([torch.arange(m, device="cuda") for m in n])
        s["out_k"] = torch.empty((L, s["cu_back"][-1], hkv, d), dtype=_DT[case["dtype"]], device="cuda")
        s["out_v"] = torch.empty_like(s["out_k"])


def _subset(gen, L, t, hkv, held, n, within=False):
    """n ascending rows for each (layer, head) of the rows that are held, of t at most,
    the last one always; heads that hold fewer have all, then -1. [L, n, hkv]."""
    score = torch.rand((L, t, hkv), generator=gen, device="cuda")
    if within:
        m = torch.tensor([x[0] for x in held], device="cuda")[:, None]
        pos = torch.arange(t, device="cuda")[None, :, None]
        score = torch.where(pos < m, score, -1.0)
        score = torch.where(pos == m - 1, 2.0, score)
    else:
        score[:, -1] = 2.0
    top = score.topk(min(n, t), dim=1)
    at = torch.where(top.values >= 0, top.indices, t).sort(dim=1).values
    at = torch.nn.functional.pad(at, (0, 0, 0, n - at.shape[1]), value=t)
    return torch.where(at < t, at, -1).to(torch.int32)


def _handles(s, case):
    """The shapes, cache, rotation and workspaces that a serving program keeps."""
    import paper_2607_22586_gb300 as M

    dt, L, kind, hq, hkv, d = int(case["dtype"] == "f32"), case["layers"], case["kind"], case["hq"], case["hkv"], case["d"]

    def shape(cu, stride_kv=0, budgets=None):
        return M.make_shape(hq, hkv, d, 2, dt, cu, budgets or [1] * (len(cu) - 1), n_layers=L, layer_stride_kv=stride_kv,
                            layer_stride_q=(len(cu) - 1) * 2 * hq * d)

    o = s["own"] = {"M": M, "rows": shape(s["cu"], s["K"].stride(0) if kind == "fork" else 0)}
    if kind == "rope":
        f, amplitude = M.rope_frequencies((case["rot"] or d), 1e6, case["scaling"], case["factor"], 32768)
        o["rotary"] = M.make_rotary(f, s["positions"], layout=case["layout"], sections=_ints(case["sections"]) or None,
                                    amplitude=amplitude)
        return
    if kind == "prompt":
        o["n"] = M.mmshift_prompt_workspace_size(o["rows"])
    else:
        o["cache"] = M.make_cache(s["kp"], s["vp"], s["table"], s["lens"], s.get("ks"), s.get("vs"))
        if kind == "shared":
            o["groups"] = list(range(0, len(s["cu"]), case["answers"]))
            o["n"] = M.mmshift_cache_shared_workspace_size(o["rows"], o["cache"], o["groups"])
        else:
            o["fill"] = shape(s["cu_fill"] if kind == "refill" else s["cu"])
            o["n"] = max(M.mmshift_cache_pages_workspace_size(o[x], o["cache"]) for x in ("rows", "fill"))
            if kind == "refill":
                o["prompt"] = shape(s["cu_seq"], s["K"].stride(0), _ints(case["rows"]))
            if "cu_back" in s:
                o["back"] = shape(s["cu_back"])
    o["ws"] = torch.zeros(o["n"], dtype=torch.uint8, device="cuda")


def _run_own(s, case):
    o, kind = s["own"], case["kind"]
    M, stream = o["M"], torch.cuda.current_stream()
    if kind == "rope":
        M.check(M.mmshift_rope(o["rows"], o["rotary"], s["Q"], s["Q"].stride(0), 0, s["K"], s["K"].stride(1), 0, s["out"],
                               s["out_k"], stream), "rope")
        return {"q": s["out"], "k": s["out_k"]}
    rest = (o["ws"], o["n"], stream)
    if kind == "prompt":
        M.check(M.mmshift_prompt_attention(o["rows"], s["Q"], s["Q"].stride(0), s["K"][0], s["V"][0], s["K"].stride(1),
                                           case["causal"], 0.0, s["out"], s["lse"], *rest), "prompt attention")
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "shared":
        M.check(M.mmshift_cache_attention_shared(o["rows"], o["cache"], o["groups"], s["Q"], s["Q"].stride(0),
                                                 case["causal"], 0.0, s["out"], s["lse"], *rest), "shared attention")
        return {"out": s["out"], "lse": s["lse"]}
    if kind in ("fork", "branch"):
        M.check(M.mmshift_cache_fork(o["rows"], o["cache"], s["refs"], s["src"], s["dst"], *rest), "fork")
    if kind == "fork":
        s["lens"].add_(s["add"])
        M.check(M.mmshift_cache_reserve(o["rows"], o["cache"], s["refs"], *rest), "reserve")
        M.check(M.mmshift_cache_append(o["rows"], o["cache"], s["K"], s["V"], s["K"].stride(1), *rest), "append")
    if kind == "refill":
        M.check(M.mmshift_cache_free(o["rows"], o["cache"], s["refs"], list(range(len(s["seq"]))), *rest), "free")
        s["lens"].copy_(s["full"])
        M.check(M.mmshift_cache_reserve(o["fill"], o["cache"], s["refs"], *rest), "reserve")
        M.check(M.mmshift_cache_fill(o["prompt"], o["cache"], s["K"], s["V"], s["idx"], None, *rest), "fill")
    if kind in ("branch", "refill"):
        M.check(M.mmshift_cache_compact(o["rows"], o["cache"], s["refs"], s["sel"], s["kept"], *rest), "compact")
    got = {"table": s["table"], "lens": s["lens"], "refs": s["refs"]}
    if "back" not in o:
        return {**got, "k": s["kp"], "v": s["vp"]}
    M.check(M.mmshift_cache_read(o["back"], o["cache"], s["first"], s["out_k"], s["out_v"], *rest), "read")
    return {**got, "k": s["out_k"], "v": s["out_v"]}


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, case)
    if kind == "rope":
        angle = s["positions"][s["axis"]].T.double() * s["freq"]
        cos, sin = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
        return {"q": _rotate(s["Q"], cos, sin, case), "k": _rotate(s["K"][0], cos, sin, case)}
    if kind == "prompt":
        return _prompt(s, case)
    if kind == "shared":
        return _attend(s, case)
    if kind in ("fork", "branch"):
        _free(s, s["dst"])
        held = (s["lens"] + case["page"] - 1) // case["page"]
        entry = torch.arange(s["table"].shape[-1], device="cuda")
        s["table"][:, s["dst"]] = torch.where(entry < held[..., None], s["table"], -1)[:, s["src"]]
        s["lens"][:, s["dst"]] = s["lens"][:, s["src"]]
        _count(s, s["table"][:, s["dst"]], 1)
    if kind == "fork":
        s["lens"].add_(s["add"])
        _reserve(s, case, s["lens"] - s["add"])
        pos = s["row_of"][None, :, None] + (s["lens"] - s["add"])[:, s["req_of"]]
        _write(s, case, s["req_of"], pos, s["K"], s["V"])
    if kind == "refill":
        _free(s, list(range(len(s["seq"]))))
        s["lens"].copy_(s["full"])
        _reserve(s, case, torch.zeros_like(s["lens"]))
        n = [b - a for a, b in zip(s["cu_fill"], s["cu_fill"][1:])]
        req = torch.repeat_interleave(torch.arange(len(n), device="cuda"), torch.tensor(n, device="cuda"))
        token = torch.tensor(s["cu_seq"], device="cuda")[req][None, :, None] + s["idx"]
        k, v = (x.gather(1, token[..., None].expand(-1, -1, -1, case["d"])) for x in (s["K"], s["V"]))
        pos = torch.cat([torch.arange(m, device="cuda") for m in n])[None, :, None].expand(token.shape)
        _write(s, case, req, pos, k, v)
    if kind in ("branch", "refill"):
        _compact(s, case)
    got = {"table": s["table"], "lens": s["lens"], "refs": s["refs"]}
    if "cu_back" not in s:
        return {**got, "k": s["kp"], "v": s["vp"]}
    pos = s["back_row"][None, :, None] + s["first"][:, s["back_req"]]
    there = pos < s["lens"][:, s["back_req"]]
    slot = _slot(s, case, s["back_req"], pos).masked_fill(~there, 0)
    return {**got, **{n: _values(s, n, slot).masked_fill(~there[..., None], 0).to(_DT[case["dtype"]]) for n in "kv"}}


def _rotate(x, cos, sin, case):
    rot, y = case["rot"] or case["d"], x.float()
    pairs = y[..., :rot].unflatten(-1, (2, rot // 2) if case["layout"] == "half" else (rot // 2, 2))
    a, b = pairs.unbind(-2 if case["layout"] == "half" else -1)
    turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -2 if case["layout"] == "half" else -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _softmax(logits, v):
    """Weighted sums of v and log-sum-exps; rows without a key give zeros and -inf."""
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    e = logits.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    return (e @ v) / total.clamp(min=1e-38), (top + total.log())[..., 0]


def _prompt(s, case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    for a, b in zip(s["cu"], s["cu"][1:]):
        n = b - a
        k, v = (s[x][0, a:b].float().transpose(0, 1)[:, None] for x in "KV")     # [hkv, 1, n, d]
        q = s["Q"][a:b].float().unflatten(1, (hkv, hq // hkv)).permute(1, 2, 0, 3)
        step = max(1, min(n, 2 ** 28 // (hq * n)))     # queries at a time: a GB of logits
        for i in range(0, n, step):
            j = min(n, i + step)
            m = j if case["causal"] else n
            z = (q[:, :, i:j] @ k[:, :, :m].transpose(-1, -2)) * d ** -0.5
            if case["causal"]:
                z.masked_fill_(torch.arange(m, device="cuda") > torch.arange(i, j, device="cuda")[:, None], -math.inf)
            o, l = _softmax(z, v[:, :, :m])
            out[a + i:a + j] = o.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
            lse[a + i:a + j] = l.permute(2, 0, 1).flatten(1, 2)
    return {"out": out, "lse": lse}


def _attend(s, case):
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    most = [int(max(x)) for x in _lens(case)[0][0]]
    for b, (a, e) in enumerate(zip(s["cu"], s["cu"][1:])):
        pos, n, lens = torch.arange(most[b], device="cuda"), e - a, s["lens"][0, b]
        slot = s["table"][0, b].long()[:, pos // page] * page + pos % page
        slot = slot.masked_fill(pos >= lens[:, None], 0)
        k, v = _values(s, "k", slot), _values(s, "v", slot).masked_fill((pos >= lens[:, None])[..., None], 0)
        q = s["Q"][a:e].float().unflatten(1, (hkv, hq // hkv)).permute(1, 0, 2, 3).flatten(1, 2)   # [hkv, n * r, d]
        z = ((q @ k.transpose(-1, -2)) * d ** -0.5).unflatten(1, (n, hq // hkv))
        limit = lens[:, None].expand(-1, n)
        if case["causal"]:
            limit = limit - n + torch.arange(1, n + 1, device="cuda")
        z.masked_fill_(pos >= limit[..., None, None], -math.inf)
        o, l = _softmax(z.flatten(1, 2), v)
        out[a:e] = o.unflatten(1, (n, -1)).permute(1, 0, 2, 3).flatten(1, 2).to(out.dtype)
        lse[a:e] = l.unflatten(1, (n, -1)).permute(1, 0, 2).flatten(1)
    return {"out": out, "lse": lse}


def _count(s, entries, by):
    e = entries[entries >= 0].long()
    s["refs"].index_add_(0, e, torch.full_like(e, by, dtype=torch.int32))


def _free(s, which):
    _count(s, s["table"][:, which], -1)
    s["table"][:, which] = -1
    s["lens"][:, which] = 0


def _take(s, need):
    """Free pages, the lowest first, for the table's entries that need one; their old pages lose a holder."""
    old = s["table"][need].long()
    got = (s["refs"] == 0).nonzero()[:len(old), 0]
    s["table"][need] = got.to(torch.int32)
    s["refs"][got] = 1
    _count(s, old, -1)
    return old, got


def _reserve(s, case, start):
    """Pages of their own for the rows from ``start`` on: missing ones, and copies of shared ones."""
    page, table = case["page"], s["table"]
    first = torch.arange(table.shape[-1], device="cuda") * page
    touched = (first < s["lens"][..., None]) & (first + page > start[..., None]) & (start < s["lens"])[..., None]
    need = touched & ((table < 0) | (s["refs"][table.clamp(min=0).long()] > 1))
    rows = (start[..., None] - first).clamp(0, page)[need]             # of a page that are there already
    old, got = _take(s, need)
    i, r = ((torch.arange(page, device="cuda") < rows[:, None]) & (old >= 0)[:, None]).nonzero(as_tuple=True)
    for name in ("kp", "vp", "ks", "vs"):
        if name in s:
            s[name][got[i], r] = s[name][old[i], r]


def _slot(s, case, req, pos, table=None):
    """The pool's row of each position [layers, rows, hkv] of the requests ``req``."""
    table = s["table"] if table is None else table
    entry = (pos // case["page"]).clamp(0, table.shape[-1] - 1).long()
    return table[:, req].gather(-1, entry[..., None])[..., 0].long() * case["page"] + pos % case["page"]


def _write(s, case, req, pos, k, v):
    there = pos < s["lens"][:, req]
    slot = _slot(s, case, req, pos)[there]
    for x, n in ((k, "k"), (v, "v")):
        if case["cache"] == "i8":
            code, scale = _quantise(x[there])
            s[n + "p"].view(-1, case["d"])[slot] = code
            s[n + "s"].view(-1)[slot] = scale
        else:
            s[n + "p"].view(-1, case["d"])[slot] = x[there]


def _compact(s, case):
    """The kept rows to the front of their sequences, the pages behind them given back."""
    page, before = case["page"], s["table"].clone()
    pages = (s["kept"] + page - 1) // page
    entry = torch.arange(before.shape[-1], device="cuda")
    mine = (s["new"] > 0)[None, :, None, None]
    _take(s, mine & (entry < pages[..., None]) & ((before < 0) | (s["refs"][before.clamp(min=0).long()] > 1)))
    there = (s["row_of"][None, :, None] < s["kept"][:, s["req_of"]])
    src = _slot(s, case, s["req_of"], s["sel"].clamp(min=0), before)[there]
    dst = _slot(s, case, s["req_of"], s["row_of"][None, :, None].expand(there.shape))[there]
    for name in ("kp", "vp", "ks", "vs"):
        if name in s:
            x = s[name].view(-1, case["d"]) if name[1] == "p" else s[name].view(-1)
            x[dst] = x[src]
    gone = mine & (entry >= pages[..., None])
    _count(s, s["table"][gone], -1)
    s["table"][gone] = -1
    s["lens"].copy_(torch.where(mine[..., 0], s["kept"], s["lens"]))


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


def work(case):
    d, hkv, hq, esz, csz, L = (case["d"], case["hkv"], case["hq"], _SIZE[case["dtype"]], _SIZE[case["cache"]],
                               case["layers"])
    kind, new, page = case["kind"], _new(case), case["page"]
    t, row = sum(new), d * csz + (4 if case["cache"] == "i8" else 0)   # a row in the pages
    if kind == "rope":
        return {"bytes": 2 * t * (hq + hkv) * d * esz + 4 * t * max(1, len(_ints(case["sections"]))),
                "flops": 3.0 * t * (hq + hkv) * (case["rot"] or d)}
    if kind == "prompt":
        pairs = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in new)
        return {"bytes": 2 * t * (hq + hkv) * d * esz + 4 * t * hq, "flops": 4.0 * d * hq * pairs}
    held, common = _lens(case)
    if kind == "shared":
        pairs = rows = 0
        for b, (unit, n) in enumerate(zip(held[0], new)):
            for m, p in zip(unit, common[b // case["answers"]]):
                pairs += n * m - (n * (n - 1) // 2 if case["causal"] else 0)
                rows += m if b % case["answers"] == 0 else m - p // page * page
        return {"bytes": 2 * row * rows + 2 * t * hq * d * esz + 4 * t * hq, "flops": 4.0 * d * (hq // hkv) * pairs}
    units = [(m, b) for layer in held for b, unit in enumerate(layer) for m in unit]
    back = 0
    if kind == "fork":
        n = _ints(case["new"])[0]
        # entries of the table written, the tail's rows copied, the new ones appended
        each = [4 * (m // page + 1) + 2 * 2 * row * (m % page) + 2 * n * (d * esz + row) for m, _ in units]
        bytes_ = case["answers"] * sum(each)
        back = case["answers"] * sum(min(m + n, page + n) for m, _ in units)
    else:
        kept = sum(min(m, _ints(case["keep"])[b]) for m, b in units)
        bytes_ = kept * (4 * row + 4)                                  # the index, the row from and to
        if kind == "refill":
            bytes_ += sum(m for m, _ in units) * (2 * (d * esz + row) + 4)
        back = kept
    if case["cache"] == "i8":
        bytes_ += 2 * back * (row + d * esz)
    return {"bytes": bytes_, "flops": 0}


def exact(case, seed):
    """Rotations, attention and 8-bit rows from their formulas in float64; counts, tables
    and copies of rows are no computed numbers."""
    kind = case["kind"]
    if kind not in ("rope", "prompt", "shared") and case["cache"] != "i8":
        return None
    s = prepare(case, seed)
    hkv, hq, d, page, cu, new = case["hkv"], case["hq"], case["d"], case["page"], s["cu"], _new(case)
    r = hq // hkv
    if kind == "rope":
        rot = case["rot"] or d
        f, amplitude = _frequencies(case)
        of = _ints(case["sections"]) or [len(f)]
        axis = [i for i, n in enumerate(of) for _ in range(n)]
        first = torch.arange(rot // 2, device="cuda") * (1 if case["layout"] == "half" else 2)
        second = first + (rot // 2 if case["layout"] == "half" else 1)
        turn = torch.polar(torch.full_like(s["positions"][axis].T, amplitude, dtype=torch.float64),
                           s["positions"][axis].T.double() * torch.tensor(f, dtype=torch.float64, device="cuda"))
        got = {}
        for name, x in (("q", s["Q"]), ("k", s["K"][0])):
            y = x.double()
            z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
            y[..., first], y[..., second] = z.real, z.imag
            got[name] = y
        return got
    if kind in ("prompt", "shared"):
        out = torch.zeros((cu[-1], hq, d), dtype=torch.float64, device="cuda")
        lse = torch.zeros((cu[-1], hq), dtype=torch.float64, device="cuda")
        lens = _lens(case)[0][0] if kind == "shared" else [[n] * hkv for n in new]
        for b, n in enumerate(new):
            for h in range(hkv):
                m = lens[b][h]
                if kind == "prompt":
                    k, v = (s[x][0, cu[b]:cu[b + 1], h].double() for x in "KV")
                else:
                    k, v = (_held(s, case, 0, b, h, m, x) for x in "kv")
                for i in range(0, n, 4096):
                    j = min(n, i + 4096)
                    end = m - n + j if case["causal"] else m
                    z = s["Q"][cu[b] + i:cu[b] + j, h * r:(h + 1) * r].double().transpose(0, 1) @ k[:end].T / math.sqrt(d)
                    if case["causal"]:
                        seen = torch.arange(end, device="cuda") <= torch.arange(m - n + i, m - n + j, device="cuda")[:, None]
                        z = torch.where(seen, z, -math.inf)
                    l = torch.logsumexp(z, -1)
                    lse[cu[b] + i:cu[b] + j, h * r:(h + 1) * r] = l.T
                    out[cu[b] + i:cu[b] + j, h * r:(h + 1) * r] = (torch.exp(z - l[..., None]) @ v[:end]).transpose(0, 1)
        return {"out": out, "lse": lse}
    # 8-bit rows that are read back, a sequence at a time
    got = {n: torch.zeros(s["out_k"].shape, dtype=torch.float64, device="cuda") for n in "kv"}
    held, rows = _lens(case)[0], len(_ints(case["rows"]))
    step = lambda x: x.abs().amax(-1, keepdim=True) / 127  # noqa: E731
    for l in range(case["layers"]):
        for b, n in enumerate(s["back"]):
            for h in range(hkv if n else 0):
                src = b if kind == "refill" else (b - rows) // case["answers"]
                m, at = held[l][src][h], s["cu_back"][b]
                for name in "kv":
                    if kind == "refill":
                        at_seq, fill = s["cu_seq"][b], s["idx"][l, s["cu_fill"][b]:s["cu_fill"][b + 1], h].long()
                        x = s[name.upper()][l, at_seq + fill, h].double()
                        x = torch.round(x / step(x)) * step(x)
                    else:
                        x = _held(s, case, l, src, h, m, name)
                    if kind == "fork":
                        y = s[name.upper()][l, cu[b]:cu[b + 1], h].double()
                        x = torch.cat([x, torch.round(y / step(y)) * step(y)])[-n:]
                    else:
                        x = x[s["sel"][l, cu[b]:cu[b] + int(min(m, new[b])), h].long()]
                    got[name][l, at:at + len(x), h] = x
    return {"table": None, "lens": None, "refs": None, **got}


def _held(s, case, l, b, h, m, name):
    """The m rows of a sequence as the pages hold them, in float64."""
    at = s["table"][l, b, h, :(m + case["page"] - 1) // case["page"]].long()
    x = s[name + "p"][at].double()
    if case["cache"] == "i8":
        x = x * s[name + "s"][at].double()[..., None]
    return x.reshape(-1, case["d"])[:m]
