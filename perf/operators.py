"""The paged K/V cache's operators: what they are measured on, and their plain forms.

A case is a dict of plain values.  `kind` names the operator:

    append   new tokens of every request: q and k are rotated by their positions, k and v go into the pages
    compact  the rows that a selection kept, all layers, from the prompt's K/V into the pages
    decode   attention of one new token per request over the pages, one layer

Pages are pools [n_pages, page, kv_heads, d] (`layout` "hnd": the same with a page's rows laid out head by head), in bf16, fp32 or
e4m3 with a scale per KV head.  A request's pages lie scattered in the pool and its last one is partly filled.

The plain forms compute in 32 bits (angles in 64) with elementary torch operations and round once at the end.
"""
import math
import random
import types

import torch

own = False

VIDEOLLAMA2 = dict(heads=32, kv_heads=8, head_dim=128, dtype="bf16", theta=10000.0, sections="", rotary=128, interleaved=False)
QWEN25VL = dict(heads=28, kv_heads=4, head_dim=128, dtype="bf16", theta=1000000.0, sections="16,24,24", rotary=128, interleaved=False)
TINY_FP32 = dict(heads=4, kv_heads=2, head_dim=64, dtype="fp32", theta=10000.0, sections="", rotary=32, interleaved=True)


def _lens(n_req, lo, hi, shape_seed=0, longest=0):
    """Requests of lo .. hi rows each; `longest`: the first one has that many instead."""
    return dict(n_req=n_req, lo=lo, hi=hi, shape_seed=shape_seed, longest=longest)


def listed():
    return [
        # One conversation's next token behind a compressed 8320-token video prompt: three position axes, latency alone.
        dict(QWEN25VL, **_lens(1, 1665, 1665), name="append_one", kind="append", cache="bf16", page=16, layout="nhd", new_lo=1, new_hi=1),
        # A token of each of 128 conversations, into an 8-bit cache.
        dict(VIDEOLLAMA2, **_lens(128, 500, 1700, 1), name="append_batch_e4m3", kind="append", cache="e4m3", page=32, layout="nhd",
             new_lo=1, new_hi=1),
        # The prompts of a ragged serving batch, one of the layers that keep every row: 8 requests of 2080 to 16640 tokens.
        dict(QWEN25VL, **_lens(8, 16700, 17000, 2), name="append_prompts", kind="append", cache="bf16", page=16, layout="nhd", new_lo=2080,
             new_hi=16640),
        # Short fp32 prompts with a partial, interleaved rotation, pages of an odd size.
        dict(TINY_FP32, **_lens(3, 310, 330, 3), name="append_fp32", kind="append", cache="fp32", page=12, layout="nhd", new_lo=37, new_hi=300),
        # The headline prompt's 26 compressed layers: 1664 of 8320 rows survive.
        dict(QWEN25VL, **_lens(1, 8320, 8320), name="compact_prompt", kind="compact", cache="bf16", page=16, layout="nhd", layers=26, keep=0.2),
        # The ragged batch's 27 layers, into an 8-bit cache.
        dict(QWEN25VL, **_lens(8, 2080, 16640, 4), name="compact_ragged_e4m3", kind="compact", cache="e4m3", page=64, layout="nhd", layers=27,
             keep=0.2),
        # One conversation over its compressed prompt: latency.
        dict(QWEN25VL, **_lens(1, 1665, 1665), name="decode_one", kind="decode", cache="bf16", page=16, layout="nhd"),
        # 128 conversations over 2900 to 5100 rows each: bandwidth.
        dict(QWEN25VL, **_lens(128, 2900, 5100, 7), name="decode_batch", kind="decode", cache="bf16", page=16, layout="nhd"),
        # The same number of conversations over an 8-bit cache laid out head by head.
        dict(VIDEOLLAMA2, **_lens(128, 2900, 5100, 8), name="decode_batch_e4m3", kind="decode", cache="e4m3", page=64, layout="hnd"),
        # One uncompressed long video among short conversations.
        dict(QWEN25VL, **_lens(64, 100, 2000, 9, longest=60000), name="decode_skewed", kind="decode", cache="bf16", page=32, layout="nhd"),
        # Two very long contexts of uncompressed layers.
        dict(VIDEOLLAMA2, **_lens(2, 150000, 250000, 10), name="decode_long", kind="decode", cache="bf16", page=64, layout="nhd"),
        # A few short fp32 conversations, pages of an odd size.
        dict(TINY_FP32, **_lens(5, 20, 700, 11), name="decode_fp32", kind="decode", cache="fp32", page=12, layout="nhd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "compact", "decode", "decode", "decode"])
    if rng.random() < 0.2:
        c = dict(TINY_FP32, cache="fp32", rotary=rng.choice([16, 32, 64]), interleaved=rng.random() < 0.5)
    else:
        c = dict(rng.choice([VIDEOLLAMA2, QWEN25VL]), cache=rng.choice(["bf16", "bf16", "e4m3"]))
        if rng.random() < 0.15:
            c.update(head_dim=64, rotary=64, sections="")
        if rng.random() < 0.3:
            group, kv = rng.choice([1, 2, 3, 5, 8, 12, 16]), rng.choice([1, 2, 3, 4, 8])
            c.update(heads=group * kv, kv_heads=kv)
    c.update(kind=kind, page=rng.choice([8, 16, 16, 32, 64, 64, 128, rng.randint(5, 100)]), layout=rng.choice(["nhd", "nhd", "hnd"]))
    n_req = 1 if rng.random() < 0.3 else _log_int(rng, 2, 160)
    seed = rng.randrange(1000)
    if kind == "append":
        if rng.random() < 0.5:  # a token of each request
            rows = _log_int(rng, 20, 5000)
            return dict(c, **_lens(n_req, max(1, rows // 2), rows, seed), new_lo=1, new_hi=1)
        n_req = min(n_req, 16)
        new = max(2, _log_int(rng, 60, min(60000, 2000000 // (c["heads"] + c["kv_heads"]))) // n_req)
        return dict(c, **_lens(n_req, new, new + rng.randint(0, 300), seed), new_lo=max(1, new // rng.randint(1, 6)), new_hi=new)
    row = c["kv_heads"] * c["head_dim"] * 2 * _bytes_of(c["cache"])  # bytes of a token's K and V
    if kind == "compact":
        n_req = min(n_req, 12)
        rows = max(20, _log_int(rng, 300, 60000) // n_req)
        return dict(c, **_lens(n_req, max(10, rows // rng.randint(1, 4)), rows, seed),
                    layers=max(1, min(rng.randint(1, 31), int(1.5e9) // (rows * n_req * row))), keep=rng.choice([0.05, 0.1, 0.2, 0.2, 0.35, 0.5]))
    rows = max(8, _log_int(rng, 200, min(500000, int(1.0e9) // row)) // n_req)
    longest = 0 if n_req == 1 or rng.random() < 0.6 else min(60000, rows * rng.randint(3, 30), int(8e9) // (n_req * c["kv_heads"] * c["head_dim"] * 4))
    return dict(c, **_lens(n_req, max(1, rows // rng.randint(1, 8)), rows, seed, longest))


# ---- the shapes a case stands for --------------------------------------------------------------------------------------
def _shape(case):
    """Rows of each request (of the prompt, for a compaction), and how many of them this call adds."""
    rng = random.Random(case["shape_seed"])
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["n_req"])]
    if case["longest"]:
        lens[0] = case["longest"]
    if case["kind"] == "compact":
        new = [max(1, int(case["keep"] * n)) for n in lens]
    elif case["kind"] == "append":
        new = [min(n, rng.randint(case["new_lo"], case["new_hi"])) for n in lens]
    else:
        new = [0] * len(lens)
    return lens, new


def _bytes_of(name):
    return {"bf16": 2, "fp32": 4, "e4m3": 1}[name]


def work(case):
    lens, new = _shape(case)
    h, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    e, ec, t = _bytes_of(case["dtype"]), _bytes_of(case["cache"]), sum(new)
    if case["kind"] == "append":  # q in and out, k and v in, k out beside the pages for prompts, k and v into the pages
        k_out = hkv if case["new_hi"] > 1 else 0
        return {"bytes": t * d * ((2 * h + 2 * hkv + k_out) * e + 2 * hkv * ec) + 4 * t * len(_axes(case)), "flops": 3.0 * t * (h + hkv) * case["rotary"]}
    if case["kind"] == "compact":
        return {"bytes": case["layers"] * t * hkv * (2 * d * (e + ec) + 4), "flops": 0.0}
    return {"bytes": sum(lens) * hkv * d * 2 * ec + 2 * len(lens) * h * d * e + 4 * sum(-(-n // case["page"]) for n in lens),
            "flops": 4.0 * sum(lens) * h * d}


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _torch_type(name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}[name]


def _axes(case):
    return [int(x) for x in case["sections"].split(",")] if case["sections"] else [case["rotary"] // 2]


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _pages(case, gen, layers, scale):
    """A pool [layers, n_pages, page, kv_heads, d] of rows that are there already; 5 % of the keys share a direction with the queries."""
    lens, new = _shape(case)
    rows = new if case["kind"] == "compact" else lens
    hkv, d, page = case["kv_heads"], case["head_dim"], case["page"]
    counts = [-(-n // page) for n in rows]
    n_pages = sum(counts) + max(2, sum(counts) // 16)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(rows), max(counts) + 1), -1, dtype=torch.int32, device="cuda")
    for r, (at, n) in enumerate(zip(_starts(counts), counts)):
        table[r, :n] = order[at:at + n]
    shape = (n_pages, page, hkv, d) if case["layout"] == "nhd" else (n_pages, hkv, page, d)
    kind = _torch_type(case["cache"])
    pools = []
    for _ in "kv":
        x = torch.empty((layers, *shape), dtype=kind, device="cuda")
        for layer in range(layers):
            for a in range(0, n_pages, 1 << 14):
                x[layer, a:a + (1 << 14)] = (_normal(gen, min(1 << 14, n_pages - a), *shape[1:]) / scale).clamp(-448.0, 448.0).to(kind)
        pools.append(x if case["layout"] == "nhd" else x.transpose(2, 3))
    return pools, table, rows


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, new = _shape(case)
    h, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    dt = _torch_type(case["dtype"])
    s = dict(case=case, n_rows=max(new if case["kind"] == "compact" else lens))
    eight = case["cache"] == "e4m3"
    layers = case.get("layers", 1)
    # what a calibration leaves: the largest value that a head showed, over the largest that the type holds
    scale = (4.5 + torch.rand((2, layers, hkv), generator=gen, device="cuda")) / 448.0 if eight else None
    (k_pages, v_pages), s["table"], rows = _pages(case, gen, layers, 5.0 / 448.0 if eight else 1.0)
    s["seq_lens"] = _ints(rows)
    if case["kind"] == "compact":
        s["k_pages"], s["v_pages"] = k_pages, v_pages
        s["k_scale"], s["v_scale"] = (scale[0], scale[1]) if eight else (None, None)
        cu, kept = _starts(lens), _starts(new)
        s["k"], s["v"] = (torch.empty((layers, cu[-1], hkv, d), dtype=dt, device="cuda") for _ in "kv")
        for x in (s["k"], s["v"]):
            for layer in range(layers):
                x[layer] = _normal(gen, cu[-1], hkv, d)
        s["idx"] = torch.empty((layers, hkv, kept[-1]), dtype=torch.int32, device="cuda")
        for r, (n, m) in enumerate(zip(lens, new)):
            chosen = torch.rand((layers, hkv, n), generator=gen, device="cuda").argsort(dim=2)[:, :, :m]
            s["idx"][:, :, kept[r]:kept[r + 1]] = chosen.sort(dim=2).values
        s["cu_seqlens"], s["cu_kept"] = _ints(cu), _ints(kept)
        return s
    s["k_pages"], s["v_pages"] = k_pages[0], v_pages[0]
    s["k_scale"], s["v_scale"] = (scale[0, 0], scale[1, 0]) if eight else (None, None)
    if case["kind"] == "decode":
        q = 1.5 * _normal(gen, len(lens), h, d)
        u = _normal(gen, hkv, d)
        u = (u / u.norm(dim=1, keepdim=True))
        q += 2.0 * u.repeat_interleave(h // hkv, dim=0)
        page, slot = torch.where(torch.rand(s["k_pages"].shape[:2], generator=gen, device="cuda") < 0.05)
        units = torch.ones(hkv, device="cuda") if s["k_scale"] is None else s["k_scale"]
        bumped = _taken(s["k_pages"], page, slot).float() * units[:, None] + 3.0 * u
        _pool(s["k_pages"])[page, slot] = _held(bumped, units, s["k_pages"].dtype)
        s["q"] = q.to(dt)
        s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty((len(lens), h), dtype=torch.float32, device="cuda")
        s["ws"] = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
        return s
    t = sum(new)
    # q, k and v are the parts of one projection's output, as a model has them
    qkv = _normal(gen, t, h + 2 * hkv, d).to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + hkv], qkv[:, h + hkv:]
    n_axes = len(_axes(case))
    # positions count the prompt's tokens, of which a compressed cache has fewer rows; further axes are a frame's rows and columns
    far = torch.cat([torch.arange(n - m, n) + 5 * n for n, m in zip(lens, new)])
    pos = torch.randint(0, 64, (n_axes, t), generator=gen, device="cuda", dtype=torch.int32)
    pos[0] = far.to(torch.int32).cuda()
    s["positions"] = pos if n_axes > 1 else pos[0]
    half = case["rotary"] // 2
    s["inv_freq"] = (case["theta"] ** (-torch.arange(half, dtype=torch.float64) / half)).cuda()
    s["sections"] = tuple(_axes(case)) if n_axes > 1 else None
    s["cu_new"] = _ints(_starts(new)) if case["new_hi"] > 1 else None
    s["q_out"] = torch.empty((t, h, d), dtype=dt, device="cuda")
    s["k_out"] = torch.empty((t, hkv, d), dtype=dt, device="cuda") if case["new_hi"] > 1 else None
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------------
def _places(s, t, cu):
    """The page and the slot in it of each of t new rows; request r's end at row seq_lens[r] of its own."""
    if cu is None:
        req, row = torch.arange(t, device="cuda"), s["seq_lens"].long() - 1
    else:
        at = torch.arange(t, device="cuda")
        req = torch.searchsorted(cu.long(), at, right=True) - 1
        row = s["seq_lens"].long()[req] - cu.long()[req + 1] + at
    page = s["k_pages"].shape[-3]
    return s["table"].long()[req, row // page], row % page, req


def _held(x, scale, kind):
    """What a pool holds for x [..., kv_heads, d]; bytes for the 8-bit type, which has no indexed stores of its own."""
    if kind is not torch.float8_e4m3fn:
        return x.to(kind)
    return (x / scale[..., None]).clamp(-448.0, 448.0).to(kind).view(torch.uint8)


def _pool(x):
    return x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x


def _taken(pool, *index):
    return _pool(pool)[index].view(pool.dtype)


def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * cos - b * sin, b * cos + a * sin
    return y


def _append_plain(s):
    case = s["case"]
    pos = s["positions"].reshape(-1, s["k"].shape[0]).double()
    axis = torch.arange(len(_axes(case))).repeat_interleave(torch.tensor(_axes(case)))
    angle = pos[axis.cuda()].T * s["inv_freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    k = _rotate(s["k"], cos, sin, case["rotary"], case["interleaved"])
    s["q_out"].copy_(_rotate(s["q"], cos, sin, case["rotary"], case["interleaved"]))
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
    page, slot, _ = _places(s, k.shape[0], s["cu_new"])
    _pool(s["k_pages"])[page, slot] = _held(k, s["k_scale"], s["k_pages"].dtype)
    _pool(s["v_pages"])[page, slot] = _held(s["v"].float(), s["v_scale"], s["v_pages"].dtype)


def _compact_plain(s):
    layers, hkv, t = s["idx"].shape
    page, slot, req = _places(s, t, s["cu_kept"])
    src = s["cu_seqlens"].long()[req] + s["idx"].long()
    layer, head = torch.arange(layers, device="cuda")[:, None, None], torch.arange(hkv, device="cuda")[:, None]
    k, v = (s[n][layer, src, head].transpose(1, 2).float() for n in "kv")
    scales = [None if s[n] is None else s[n][:, None] for n in ("k_scale", "v_scale")]
    _pool(s["k_pages"])[:, page, slot] = _held(k, scales[0], s["k_pages"].dtype)
    _pool(s["v_pages"])[:, page, slot] = _held(v, scales[1], s["v_pages"].dtype)


def _decode_plain(s):
    q, lens, page = s["q"].float(), s["seq_lens"].long(), s["k_pages"].shape[1]
    n_req, h, d = q.shape
    hkv = s["k_pages"].shape[2]
    row = torch.arange(s["n_rows"], device="cuda")
    pages = s["table"].long()[:, row // page].clamp(min=0)
    there = row < lens[:, None]
    k = _taken(s["k_pages"], pages, row % page).float()
    logits = torch.einsum("rghd,rlgd->rghl", q.view(n_req, hkv, h // hkv, d) / math.sqrt(d), k)
    del k
    if s["k_scale"] is not None:
        logits *= s["k_scale"][:, None, None]
    logits = torch.where(there[:, None, None], logits, -math.inf)
    top = logits.amax(dim=3, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(dim=3, keepdim=True)
    o = torch.einsum("rghl,rlgd->rghd", p, _taken(s["v_pages"], pages, row % page).float()) / total
    if s["v_scale"] is not None:
        o *= s["v_scale"][:, None, None]
    s["o"].copy_(o.reshape(n_req, h, d))
    s["lse"].copy_((top + torch.log(total)).reshape(n_req, h))


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2510_25600_b200 import binding as P
        if kind == "append":
            P.purekv_append_paged(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["seq_lens"], s["cu_new"], q=s["q"], q_out=s["q_out"],
                                  k_out=s["k_out"], positions=s["positions"], inv_freq=s["inv_freq"], sections=s["sections"],
                                  interleaved=case["interleaved"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        elif kind == "compact":
            batch = types.SimpleNamespace(cu_seqlens=s["cu_seqlens"])
            budget = types.SimpleNamespace(cu_kept=s["cu_kept"])
            P.purekv_compact_paged(s["k"], s["v"], s["idx"], batch, budget, s["k_pages"], s["v_pages"], s["table"], s["seq_lens"],
                                   k_scale=s["k_scale"], v_scale=s["v_scale"])
        else:
            P.purekv_decode_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["seq_lens"], max_len=s["n_rows"], out=s["o"], lse=s["lse"],
                                  k_scale=s["k_scale"], v_scale=s["v_scale"], ws=s["ws"])
    else:
        {"append": _append_plain, "compact": _compact_plain, "decode": _decode_plain}[kind](s)
    if kind == "decode":
        return {"o": s["o"], "lse": s["lse"]}
    out = {"k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    if kind == "append":
        out["q"] = s["q_out"]
        if s["k_out"] is not None:
            out["k"] = s["k_out"]
    return out


# ---- the definitions in 64 bits, request by request ----------------------------------------------------------------------
def _rows_of(s, r, n):
    page = s["k_pages"].shape[-3]
    row = torch.arange(n, device="cuda")
    return s["table"][r].long()[row // page] * page + row % page


def _flat(pool):
    """[..., n_pages, page, kv_heads, d] in 64 bits with pages and slots as one axis."""
    return pool.double().flatten(-4, -3)


def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _shape(case)
    h, hkv, d = case["heads"], case["kv_heads"], case["head_dim"]
    ks = s["k_scale"].double() if s["k_scale"] is not None else torch.ones(hkv, dtype=torch.float64, device="cuda")
    vs = s["v_scale"].double() if s["v_scale"] is not None else torch.ones(hkv, dtype=torch.float64, device="cuda")
    if case["kind"] == "decode":
        o = torch.empty((len(lens), h, d), dtype=torch.float64, device="cuda")
        lse = torch.empty((len(lens), h), dtype=torch.float64, device="cuda")
        for r, n in enumerate(lens):
            at = _rows_of(s, r, n)
            for g in range(hkv):
                k = _taken(s["k_pages"][:, :, g], at // case["page"], at % case["page"]).double() * ks[g]
                v = _taken(s["v_pages"][:, :, g], at // case["page"], at % case["page"]).double() * vs[g]
                heads = slice(g * (h // hkv), (g + 1) * (h // hkv))
                z = s["q"][r, heads].double() @ k.T / d ** 0.5
                lse[r, heads] = torch.logsumexp(z, dim=1)
                o[r, heads] = torch.softmax(z, dim=1) @ v
        return {"o": o, "lse": lse}
    eight = case["cache"] == "e4m3"
    k_pages, v_pages = _flat(s["k_pages"]), _flat(s["v_pages"])
    shape = s["k_pages"].shape
    clamp = (lambda x: x.clamp(-448.0, 448.0)) if eight else (lambda x: x)
    out, at = {}, 0
    if case["kind"] == "compact":
        base = 0
        for r, (n, m) in enumerate(zip(lens, new)):
            rows = _rows_of(s, r, m)
            for layer in range(case["layers"]):
                for g in range(hkv):
                    src = base + s["idx"][layer, g, at:at + m].long()
                    ku, vu = (ks[layer, g], vs[layer, g]) if eight else (1.0, 1.0)
                    k_pages[layer, rows, g] = clamp(s["k"][layer, src, g].double() / ku)
                    v_pages[layer, rows, g] = clamp(s["v"][layer, src, g].double() / vu)
            base, at = base + n, at + m
        return {"k_pages": k_pages.view(shape), "v_pages": v_pages.view(shape)}
    rot, pos = case["rotary"], s["positions"].reshape(-1, sum(new)).double()
    table, axis = [], 0
    for count in _axes(case):
        table += [axis] * count
        axis += 1
    out["q"] = s["q"].double().clone()
    k = s["k"].double().clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + rot // 2)
        turn = torch.exp(1j * pos[table[i]] * case["theta"] ** (-2.0 * i / rot))[:, None]
        for x in (out["q"], k):
            z = torch.complex(x[..., a], x[..., b]) * turn
            x[..., a], x[..., b] = z.real, z.imag
    for r, (n, m) in enumerate(zip(lens, new)):
        rows = _rows_of(s, r, n)[n - m:]
        k_pages[rows] = clamp(k[at:at + m] / ks[:, None])
        v_pages[rows] = clamp(s["v"][at:at + m].double() / vs[:, None])
        at += m
    out.update(k_pages=k_pages.view(shape), v_pages=v_pages.view(shape))
    if s["k_out"] is not None:
        out["k"] = k
    return out
