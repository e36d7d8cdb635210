"""Cases of the 4-bit cache and page operators: inputs, plain forms and the library's calls.

A 4-bit pool holds K and V as uint8 [pages][2][Hkv][P * (D / 2 + D / 16)]: P rows of D / 2 bytes, two e2m1 values each (the
even element in the low half), then P rows of D / 16 e4m3 scales, one for 16 neighbouring elements.  A value stands for
e2m1 * scale * g with one g for a layer's K and one for its V.

  append   the step's K/V rows rounded into the pool, and read back as the cache now holds them
  attn     softmax(scale q K^T) V over a 4-bit cache, causal within the step (whose rows are held already) or not
  fork     the block tables of a step's rows from those of their parents: shared, passed on, fresh and freed pages
  compact  pages of high number moved into the lowest free ones: counts, tables, page map and moves
  copy     page pairs copied in every layer's pool
"""
import math
import random

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def _case(name, op, **more):
    c = {"op": op, **more}
    if name:
        c["name"] = name
    return c


def _heads(hq, hkv, d, page):
    return {"hq": hq, "hkv": hkv, "d": d, "page": page}


def listed():
    big, small = _heads(64, 8, 128, 64), _heads(4, 1, 64, 16)
    return [
        # a decode step of a full batch: one row per request
        _case("append_decode_b64", "append", **big, batch=64, lo=4096, hi=32768, q_lo=1, q_hi=1, k_scale=1.0, v_scale=0.5),
        # prompts of ragged lengths, some behind a cached prefix
        _case("append_prompt_b8", "append", **big, batch=8, lo=0, hi=4099, q_lo=1, q_hi=8192, k_scale=0.046875, v_scale=1.0),
        # two requests, one token each, short contexts: nothing but launch latency
        _case("attn_decode_tiny", "attn", **small, batch=2, lo=100, hi=512, q_lo=1, q_hi=1, causal=True, k_scale=1.0, v_scale=1.0),
        # a full decode batch at the serving heads: the stream of 4-bit rows
        _case("attn_decode_b64", "attn", **big, batch=64, lo=4096, hi=32768, q_lo=1, q_hi=1, causal=True, k_scale=1.0, v_scale=0.5),
        # two to four tokens per request (drafts to be checked)
        _case("attn_draft_b32", "attn", **big, batch=32, lo=4096, hi=32768, q_lo=2, q_hi=4, causal=True, k_scale=0.046875, v_scale=1.0),
        # chunks of prompts behind cached prefixes that may be empty: the matrix products
        _case("attn_prompt_b8", "attn", **big, batch=8, lo=0, hi=8192, q_lo=257, q_hi=512, causal=True, k_scale=1.0, v_scale=1.0),
        # a small server's beams
        _case("fork_b8", "fork", page=16, rows=8, parents=8, hi=512, pages=2048, beam=True, extra=16),
        # a large server's step: most rows go on, some fork, some end, the pool of a whole card
        _case("fork_b512", "fork", page=64, rows=512, parents=480, hi=131072, pages=1000003, beam=False, extra=129),
        # a small pool
        _case("compact_2k", "compact", page=16, rows=8, hi=512, pages=2048, moves=256, live=0.3),
        # the pool of a whole card, long tables
        _case("compact_1m", "compact", page=64, rows=512, hi=131072, pages=1000003, moves=4096, live=0.6),
        # the partly filled pages of a few forked rows in two layers
        _case("copy_l2", "copy", hkv=4, d=128, page=32, pages=64, pairs=5, layers=2),
        # a step's pairs in a stack of layers
        _case("copy_l10", "copy", hkv=8, d=128, page=64, pages=512, pairs=200, layers=10),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "fork", "compact", "copy"])
    page = rng.choice([16, 32, 64, 64])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 3, 4, 8])
    if op in ("append", "attn"):
        group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8])
        hi = _log_int(rng, 48, 32768)
        lo = rng.choice([0, rng.randint(0, hi // 2), rng.randint(hi // 2, hi)])
        batch = _log_int(rng, 1, 64)
        q_hi = rng.choice([1, rng.randint(2, 8), _log_int(rng, 2, 512)])
        q_lo = q_hi if q_hi == 1 else rng.randint(0, q_hi)
        # no more than the largest listed case: padded scores and cached rows
        while batch > 1 and (batch * q_hi * (hi + q_hi) * group * hkv > 1.5e9 or batch * hi * hkv * d > 1.5e9):
            batch = max(1, batch // 2)
        while q_hi * (hi + q_hi) * group * hkv > 1.5e9:
            hi //= 2
            lo = min(lo, hi)
        more = {"causal": rng.random() < 0.75} if op == "attn" else {}
        return _case(None, op, **_heads(group * hkv, hkv, d, page), batch=batch, lo=lo, hi=hi, q_lo=q_lo, q_hi=q_hi,
                     k_scale=rng.choice([1.0, 0.25, 0.046875]), v_scale=rng.choice([1.0, 0.25, 0.046875]), **more)
    if op == "copy":
        pairs = _log_int(rng, 1, 400)
        layers = _log_int(rng, 1, 40)
        while pairs * layers * hkv * d * page > 200 * 10 * 8 * 128 * 64 and pairs > 1:
            pairs = max(1, pairs // 2)
        return _case(None, op, hkv=hkv, d=d, page=page, pages=2 * pairs + rng.randint(1, 50), pairs=pairs, layers=layers)
    rows = _log_int(rng, 1, 512)
    hi = _log_int(rng, 1, 131072)
    pages = min(1000003, rows * (-(-hi // page) + 4) * 2 + _log_int(rng, 100, 200000))
    while rows * (-(-hi // page) + 4) > 0.3 * pages and rows > 1:
        rows //= 2
    if op == "fork":
        return _case(None, op, page=page, rows=rows, parents=max(1, rows + rng.randint(-rows // 4, rows // 4)), hi=hi, pages=pages,
                     beam=rng.random() < 0.5, extra=rng.randint(1, 3 * page))
    return _case(None, op, page=page, rows=rows, hi=hi, pages=pages, moves=_log_int(rng, 1, 8192), live=rng.choice([0.35, 0.6, 0.9]))


def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lens(case):
    """(cached length, new tokens) of each request: of the case alone, the same for every seed."""
    rng = _rng(case)
    b = case["batch"]
    ctx = [rng.randint(case["lo"], case["hi"]) for _ in range(b)]
    ctx[rng.randrange(b)] = case["hi"]
    if b > 2:
        ctx[0] = case["lo"]  # the shortest one; an empty one where the range has it
    q = [rng.randint(case["q_lo"], case["q_hi"]) for _ in range(b)]
    q[-1] = case["q_hi"]
    return ctx, q


def _rows(case):
    """Token lengths of the rows that hold pages, and for a fork each new row's (parent, length, room)."""
    rng = _rng(case)
    n = case.get("parents", case["rows"])
    have = [rng.randint(0, case["hi"]) for _ in range(n)]
    have[rng.randrange(n)] = case["hi"]
    made = []
    for r in range(case["rows"] if case["op"] == "fork" else 0):
        p = rng.randrange(n) if case["beam"] else (r if r < n and rng.random() < 0.9 else rng.choice([-1, rng.randrange(n)]))
        length = 0 if p < 0 else max(0, have[p] - rng.choice([0, 0, 0, rng.randint(0, 4)]))
        made.append((p, length, length + rng.randint(0, case["extra"])))
    return have, made


def work(case):
    op = case["op"]
    if op in ("append", "attn"):
        ctx, q = _lens(case)
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        row = 2 * hkv * d * 9 // 16  # K and V of a position
        if op == "append":
            new = sum(q)
            return {"bytes": new * (2 * row + 8 * hkv * d), "flops": 4 * new * hkv * d}
        seen = [(n, c + (n if case["causal"] else 0)) for n, c in zip(q, ctx) if n]
        pairs = sum(n * c + (n * (n + 1) // 2 if case["causal"] else 0) for n, c in zip(q, ctx))
        return {"bytes": row * sum(c for _, c in seen) + sum(q) * hq * (4 * d + 4), "flops": 4 * pairs * hq * d}
    if op == "copy":
        return {"bytes": 2 * case["pairs"] * case["layers"] * 2 * case["hkv"] * case["page"] * case["d"] * 2, "flops": 0}
    have, made = _rows(case)
    held = sum(-(-n // case["page"]) for n in have)
    if op == "fork":
        new = sum(-(-max(n, m) // case["page"]) for _, n, m in made)
        return {"bytes": 4 * (2 * case["pages"] + held + new), "flops": 0}
    return {"bytes": 4 * (3 * case["pages"] + 2 * held + 2 * case["moves"]), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _tables(used, blocks, perm):
    """Block tables whose row r holds the next used[r] entries of perm; the places behind hold -1."""
    b = len(used)
    counts = torch.tensor(used, device="cuda")
    start = torch.cumsum(counts, 0) - counts
    at = torch.arange(blocks, device="cuda")[None, :]
    inside = at < counts[:, None]
    return torch.where(inside, perm[(start[:, None] + at).clamp_(max=perm.numel() - 1)], -1).to(torch.int32).reshape(b, blocks).contiguous()


def _levels(dtype):
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=dtype, device="cuda")
    return torch.cat([v, -v])


def _round4(x, g):
    """x [..., D] in 32 bits -> bytes [..., D / 2] and scale bytes [..., D / 16]."""
    t = x.reshape(*x.shape[:-1], -1, 16)
    f = ((t.abs().amax(dim=-1) / g) / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    s = (f.float() * g)[..., None]
    # 64 bits: a value halfway between two levels has to come out as one
    y = torch.where(s > 0, t.abs().double() / s.double(), 0.0)
    # ties go to the level of even code
    n = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)).to(torch.uint8)
    n = (n + 8 * (torch.signbit(t) & (s > 0)).to(torch.uint8)).reshape(x.shape)
    return n[..., 0::2] + 16 * n[..., 1::2], f.view(torch.uint8)


def _filled(pages, hkv, page, d, k_scale, v_scale, g):
    """A pool whose every row was rounded from normal values."""
    pool = torch.empty((pages, 2, hkv, page * (d // 2 + d // 16)), dtype=torch.uint8, device="cuda")
    step = max(1, 1 << 25 >> (hkv * page * d).bit_length())
    for i in range(0, pages, step):
        n = min(step, pages - i)
        for which, scale in ((0, k_scale), (1, v_scale)):
            data, f = _round4(torch.randn((n, hkv, page, d), generator=g, device="cuda"), scale)
            pool[i:i + n, which] = torch.cat([data.reshape(n, hkv, -1), f.reshape(n, hkv, -1)], dim=-1)
    return pool


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, page = case["op"], case["page"]
    s = {"case": case}
    if op in ("append", "attn"):
        ctx, q_len = _lens(case)
        b, hq, hkv, d = (case[k] for k in ("batch", "hq", "hkv", "d"))
        s.update(ctx=_i32(ctx), max_ctx=max(ctx), q_len=q_len, total_q=sum(q_len), max_q=max(q_len), scale=1.0 / math.sqrt(d))
        s["indptr"] = _i32([sum(q_len[:r]) for r in range(b + 1)])
        s["req"] = torch.tensor([r for r in range(b) for _ in range(q_len[r])], dtype=torch.int64, device="cuda")
        s["tok"] = torch.tensor([i for r in range(b) for i in range(q_len[r])], dtype=torch.int64, device="cuda")
        # pages of a request in any order; the slots behind its last row hold what an earlier request left there
        rows = [c + (n if op == "append" or case["causal"] else 0) for c, n in zip(ctx, q_len)]
        used = [-(-n // page) for n in rows]
        pages = sum(used) + 1
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = _tables(used, max(1, max(used)), perm)
        s["table"] = torch.where(table < 0, perm[-1], table).contiguous()
        total = s["total_q"]
        if op == "append":
            s["pool"] = torch.randint(0, 127, (pages, 2, hkv, page * (d // 2 + d // 16)), generator=g, device="cuda", dtype=torch.uint8)
            s["k"], s["v"] = (torch.randn((total, hkv, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            s["k_out"], s["v_out"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        else:
            s["pool"] = _filled(pages, hkv, page, d, case["k_scale"], case["v_scale"], g)
            s["q"] = torch.randn((total, hq, d), generator=g, device="cuda", dtype=torch.bfloat16)
            s["out"] = torch.zeros((total, hq, d), dtype=torch.bfloat16, device="cuda")
            s["lse"] = torch.zeros((total, hq), dtype=torch.float32, device="cuda")
    elif op == "copy":
        n, pairs = case["pages"], case["pairs"]
        s["pools"] = [torch.randn((n, 2, case["hkv"], page, case["d"]), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(case["layers"])]
        perm = torch.randperm(n, generator=g, device="cuda").to(torch.int32)
        # a list of fixed length: the places behind the step's pairs hold -1; a page may be copied to several
        src = perm[torch.randint(0, max(1, pairs - 1), (pairs,), generator=g, device="cuda")]
        none = torch.full((max(1, pairs // 4),), -1, dtype=torch.int32, device="cuda")
        s["src"], s["dst"] = torch.cat([src, none]), torch.cat([perm[pairs:2 * pairs], none])
    else:
        have, made = _rows(case)
        pages = case["pages"]
        held = [-(-n // page) for n in have]
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        blocks = max(1, max(held), max([-(-max(n, m) // page) for _, n, m in made] or [1]))
        s["table"] = _tables(held, blocks, perm)
        s["held"] = _i32(held)
        ref = torch.zeros((pages,), dtype=torch.int32, device="cuda")
        ref[perm[: sum(held)].long()] = 1
        if op == "fork":
            # a prefix cache holds a tenth of the rows' pages and pages of its own
            more = torch.rand((pages,), generator=g, device="cuda")
            ref += (more < 0.1).to(torch.int32)
            s["parent"], s["length"], s["need"] = (_i32([m[i] for m in made]) for i in range(3))
            n = len(made)
            s["table_out"] = torch.full((n, blocks), -1, dtype=torch.int32, device="cuda")
            s["held_out"], s["copy_src"], s["copy_dst"] = (torch.zeros((n,), dtype=torch.int32, device="cuda") for _ in range(3))
        else:
            ref += (torch.rand((pages,), generator=g, device="cuda") < case["live"]).to(torch.int32)
            s["table_out"] = torch.full_like(s["table"], -1)
            s["page_map"] = torch.zeros_like(ref)
            s["move_src"], s["move_dst"] = (torch.zeros((case["moves"],), dtype=torch.int32, device="cuda") for _ in range(2))
        s["ref"], s["ref_out"] = ref, torch.zeros_like(ref)
    if own:
        _open(s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------------------------------------------------
_handles = {}


def _open(s):
    """The handle, layers, batch and workspace that a user's program keeps."""
    from paper_2607_13095_b200 import binding as hb
    c = s["case"]
    key = (c.get("hq", c.get("hkv", 1)), c.get("hkv", 1), c.get("d", 128), c["page"])
    if key not in _handles:
        _handles[key] = hb.Handle(*key, out_dtype=torch.bfloat16)
    s["hb"], s["h"] = hb, _handles[key]
    if c["op"] in ("append", "attn"):
        s["layer"] = hb.PackedLayer(s["pool"], c["k_scale"], c["v_scale"])
        ring = torch.zeros((c["batch"], s["h"].ring_pages), dtype=torch.int32, device="cuda")
        head = torch.zeros((c["batch"],), dtype=torch.int32, device="cuda")
        one = c["q_lo"] == 1 and c["q_hi"] == 1
        s["batch"] = hb.Batch(s["ctx"], s["table"], ring, head, None if one else s["indptr"], max_q_len=s["max_q"], total_q=s["total_q"],
                              max_ctx_len=s["max_ctx"])
    if c["op"] == "attn":
        need = hb.hswa_packed_workspace_need(s["h"], c["batch"], s["total_q"], s["max_q"], s["max_ctx"], c["causal"])
        s["ws"] = torch.empty((max(need, 256),), dtype=torch.uint8, device="cuda")
    if c["op"] == "fork":
        s["ws"] = torch.empty((hb.hswa_pages_workspace_need(s["h"], c["pages"]),), dtype=torch.uint8, device="cuda")
    if c["op"] == "copy":
        s["layers"] = [hb.Layer(p, False) for p in s["pools"]]


def _run_own(s):
    hb, c, h = s["hb"], s["case"], s["h"]
    if c["op"] == "append":
        hb.hswa_packed_append(h, s["layer"], s["batch"], s["k"], s["v"])
        hb.hswa_packed_read(h, s["layer"], s["batch"], s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if c["op"] == "attn":
        hb.hswa_packed_attn(h, s["layer"], s["batch"], c["causal"], s["q"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "fork":
        hb.hswa_pages_fork(h, s["ref"], s["ref_out"], s["table"], s["held"], s["parent"], s["length"], s["need"], s["table_out"],
                           s["held_out"], s["copy_src"], s["copy_dst"], s["ws"])
        return _fork_outputs(s)
    if c["op"] == "compact":
        hb.hswa_pages_compact(h, s["ref"], s["ref_out"], s["table"], s["held"], s["table_out"], s["page_map"], s["move_src"], s["move_dst"])
        return _compact_outputs(s)
    hb.hswa_pages_copy(h, s["layers"], s["src"], s["dst"])
    return s["pools"]


def _fork_outputs(s):
    return {k: s[k] for k in ("ref_out", "table_out", "held_out", "copy_src", "copy_dst")}


def _compact_outputs(s):
    return {k: s[k] for k in ("ref_out", "table_out", "page_map", "move_src", "move_dst")}


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _split(s, slabs):
    """Slabs [..., P * (D / 2 + D / 16)] -> bytes [..., P, D / 2] and scales [..., P, D / 16]."""
    c = s["case"]
    p, d = c["page"], c["d"]
    return slabs[..., : p * d // 2].unflatten(-1, (p, d // 2)), slabs[..., p * d // 2:].unflatten(-1, (p, d // 16))


def _values(data, f, g):
    """Bytes [..., D / 2] and scale bytes [..., D / 16] -> the values they stand for, [..., D] in 32 bits."""
    v = _levels(torch.float32)
    both = torch.stack([v[(data & 15).int()], v[(data >> 4).int()]], dim=-1).flatten(-2)
    scale = f.contiguous().view(torch.float8_e4m3fn).float() * g
    return (both.unflatten(-1, (-1, 16)) * scale[..., None]).flatten(-2)


def _plain_append(s):
    c = s["case"]
    pos = s["ctx"].long()[s["req"]] + s["tok"]
    pages, slot = s["table"][s["req"], pos // c["page"]].long(), pos % c["page"]
    outs = {}
    for which, name, g in ((0, "k", c["k_scale"]), (1, "v", c["v_scale"])):
        data, f = _split(s, s["pool"][:, which])  # views of the pool
        head = torch.arange(c["hkv"], device=slot.device)
        new, new_f = _round4(s[name].float(), g)
        data[pages[:, None], head, slot[:, None]] = new
        f[pages[:, None], head, slot[:, None]] = new_f
        outs[name] = _values(data[pages[:, None], head, slot[:, None]], f[pages[:, None], head, slot[:, None]], g).to(torch.bfloat16)
    return outs


def _gather(s, which, g):
    """The cached K (0) or V (1) of every request, padded: [B][Hkv][L][D] in 32 bits."""
    data, f = _split(s, s["pool"][s["table"].long(), which])  # [B][blocks][Hkv][P][...]
    t = _values(data.transpose(1, 2), f.transpose(1, 2), g)
    return t.flatten(2, 3)


def _pad_rows(s, x):
    """[T][Hq][D] -> [B][Hkv][tokens * G][D], padded to the longest request."""
    c = s["case"]
    grp = c["hq"] // c["hkv"]
    y = torch.zeros((c["batch"], s["max_q"], *x.shape[1:]), dtype=torch.float32, device=x.device)
    y[s["req"], s["tok"]] = x.float()
    return y.unflatten(2, (c["hkv"], grp)).transpose(1, 2).flatten(2, 3)


def _unpad_rows(s, y):
    """[B][Hkv][tokens * G][...] -> [T][Hq][...]"""
    c = s["case"]
    grp = c["hq"] // c["hkv"]
    y = y.unflatten(2, (s["max_q"], grp)).transpose(1, 2).flatten(2, 3)
    return y[s["req"], s["tok"]]


def _plain_attn(s):
    c = s["case"]
    k = _gather(s, 0, c["k_scale"])
    sc = (_pad_rows(s, s["q"]) * s["scale"]) @ k.transpose(2, 3)
    del k
    j = torch.arange(sc.shape[-1], device=sc.device)
    end = s["ctx"].long()[:, None].expand(-1, sc.shape[2])
    if c["causal"]:
        end = end + torch.arange(s["max_q"], device=sc.device).repeat_interleave(c["hq"] // c["hkv"])[None, :] + 1
    sc.masked_fill_(j >= end[:, None, :, None], -math.inf)
    m = sc.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(sc - m)
    del sc
    total = e.sum(dim=-1, keepdim=True)
    lse = (m + torch.log(total))[..., 0]
    out = torch.where(total > 0, (e @ _gather(s, 1, c["v_scale"])) / total, 0.0)
    return {"out": _unpad_rows(s, out).to(torch.bfloat16), "lse": _unpad_rows(s, lse).contiguous()}


def _plain_fork(s):
    p = s["case"]["page"]
    ref, table, held, parent, length, need = s["ref"], s["table"], s["held"], s["parent"].long(), s["length"], s["need"]
    n, blocks = s["table_out"].shape
    pages = ref.numel()
    from_row = parent.clamp(min=0)
    child = parent >= 0
    rows = torch.arange(n, device=ref.device)
    first = torch.full((held.numel(),), n, device=ref.device).scatter_reduce(0, from_row, torch.where(child, rows, n), "amin")
    most = torch.zeros_like(first).scatter_reduce(0, from_row, torch.where(child, length // p, 0).long(), "amax")
    is_first = child & (first[from_row] == rows)
    k = torch.arange(blocks, device=ref.device)[None, :]
    full = (length // p)[:, None]
    held_out = torch.maximum(-(-length // p), -(-need // p))
    src = torch.nn.functional.pad(table, (0, max(0, blocks - table.shape[1])), value=-1)[from_row, :blocks]
    have = child[:, None] & (k < held[from_row][:, None])
    shared = have & (k < full)
    # a page that the parent alone holds, and that none of its children shares, goes on to its first child
    passed = have & (k >= most[from_row][:, None]) & (k < held_out[:, None]) & is_first[:, None] & (ref[src.clamp(min=0).long()] == 1)
    fresh = (k < held_out[:, None]) & ~shared & ~passed
    free = ref == 0
    order = torch.full((pages + 1,), -1, dtype=torch.int32, device=ref.device)
    order.scatter_(0, torch.where(free, torch.cumsum(free, 0) - 1, pages), torch.arange(pages, dtype=torch.int32, device=ref.device))
    rank = (torch.cumsum(fresh.flatten(), 0) - 1).reshape(fresh.shape).clamp(min=0, max=pages)
    taken = torch.where(fresh, order[rank], src)
    s["table_out"].copy_(torch.where(k < held_out[:, None], taken, s["table_out"]))
    s["held_out"].copy_(held_out)
    tail = (k == full) & (length % p != 0)[:, None] & fresh
    s["copy_src"].copy_(torch.where(tail, src, -1).amax(dim=1))
    s["copy_dst"].copy_(torch.where(tail, taken, -1).amax(dim=1))
    at = torch.arange(table.shape[1], device=ref.device)[None, :] < held[:, None]
    count = torch.cat([ref, ref.new_zeros(1)])
    count.scatter_add_(0, torch.where(at, table, pages).long().flatten(), torch.where(at, -1, 0).to(torch.int32).flatten())
    inside = k < held_out[:, None]
    count.scatter_add_(0, torch.where(inside, taken, pages).long().flatten(), inside.to(torch.int32).flatten())
    s["ref_out"].copy_(count[:pages])
    return _fork_outputs(s)


def _plain_compact(s):
    ref, table, held = s["ref"], s["table"], s["held"]
    pages, most = ref.numel(), s["move_src"].numel()
    live = ref > 0
    total = live.sum()
    at = torch.arange(pages, dtype=torch.int32, device=ref.device)
    hole = ~live & (at < total)
    high = live & (at >= total)
    n = hole.sum()  # holes below the number of live pages, as many as live pages from there on
    from_low = torch.cumsum(hole, 0) - 1
    from_high = n - torch.cumsum(high, 0)
    src = torch.full((most + 1,), -1, dtype=torch.int32, device=ref.device)
    dst = src.clone()
    dst.scatter_(0, torch.where(hole & (from_low < most), from_low, most), at)
    src.scatter_(0, torch.where(high & (from_high < most), from_high, most), at)
    s["move_src"].copy_(src[:most])
    s["move_dst"].copy_(dst[:most])
    moved = high & (from_high < most)
    s["page_map"].copy_(torch.where(moved, dst[torch.where(moved, from_high, most)], at))
    took = hole & (from_low < most)
    s["ref_out"].copy_(torch.where(moved, 0, torch.where(took, ref[src[torch.where(took, from_low, most)].clamp(min=0).long()], ref)))
    at = torch.arange(table.shape[1], device=ref.device)[None, :] < held[:, None]
    s["table_out"].copy_(torch.where(at, s["page_map"][table.clamp(min=0).long()], s["table_out"]))
    return _compact_outputs(s)


def _plain_copy(s):
    n = s["case"]["pairs"]
    src, dst = s["src"][:n].long(), s["dst"][:n].long()
    for pool in s["pools"]:
        pool[dst] = pool[src]
    return s["pools"]


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "attn": _plain_attn, "fork": _plain_fork, "compact": _plain_compact, "copy": _plain_copy}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_rounded(x, g):
    """[T][Hkv][D] -> the values that the cache holds for them, by the nearest of all levels."""
    t = x.double().reshape(*x.shape[:-1], -1, 16)
    codes = torch.arange(0, 127, device=x.device, dtype=torch.uint8).view(torch.float8_e4m3fn).double()  # 0 .. 448, ascending
    want = t.abs().amax(dim=-1, keepdim=True) / g / 6.0
    hi = torch.searchsorted(codes, want.contiguous()).clamp(min=1, max=126)
    lo = hi - 1
    below, above = want - codes[lo], codes[hi] - want
    at = torch.where(below < above, lo, torch.where(above < below, hi, torch.where(lo % 2 == 0, lo, hi)))
    scale = codes[at] * g
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    best = torch.zeros_like(t)
    off = torch.full_like(t, math.inf)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):  # the even ones first: they win ties
        d = (t.abs() - levels[code] * scale).abs()
        best = torch.where(d < off, levels[code], best)
        off = torch.minimum(off, d)
    return (torch.sign(t) * best * scale).reshape(x.shape)


def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None
    s = prepare(case, seed)
    if case["op"] == "copy":
        whole = [p.double() for p in s["pools"]]
        for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
            for new, old in zip(whole if a >= 0 else [], s["pools"]):
                new[b] = old[a].double()
        return whole
    if case["op"] == "append":
        return {"k": _exact_rounded(s["k"], case["k_scale"]), "v": _exact_rounded(s["v"], case["v_scale"])}
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    g = hq // hkv
    ctx, q_len = _lens(case)
    out = torch.zeros((sum(q_len), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((sum(q_len), hq), -math.inf, dtype=torch.float64, device="cuda")
    levels = _levels(torch.float64)
    t0 = 0
    for r in range(case["batch"]):
        c, n = ctx[r], q_len[r]
        total = c + n if case["causal"] else c
        pos = torch.arange(total, device="cuda")
        slabs = s["pool"][s["table"][r].long()[pos // page]]  # [total][2][Hkv][...]
        at = (pos % page)[:, None, None, None]
        both = []
        for which, scale in ((0, case["k_scale"]), (1, case["v_scale"])):
            i = torch.arange(d, device="cuda")
            byte = slabs[:, which].gather(2, (at[..., 0] * (d // 2) + i // 2).expand(total, hkv, d))
            code = (byte.int() >> (4 * (i % 2)).int()) & 15
            f = slabs[:, which].gather(2, (page * d // 2 + at[..., 0] * (d // 16) + i // 16).expand(total, hkv, d))
            both.append(levels[code] * f.contiguous().view(torch.float8_e4m3fn).double() * scale)
        k, v = both
        step = max(1, int(1e8 // max(1, total * hq)))
        for i0 in range(0, n if total else 0, step):
            i1 = min(n, i0 + step)
            q = s["q"][t0 + i0:t0 + i1].double().reshape(i1 - i0, hkv, g, -1)
            sc = torch.einsum("ihgd,jhd->hgij", q, k) / math.sqrt(d)
            if case["causal"]:
                late = torch.arange(total, device="cuda")[None, :] > c + torch.arange(i0, i1, device="cuda")[:, None]
                sc = sc.masked_fill(late, -math.inf)
            out[t0 + i0:t0 + i1] = torch.einsum("hgij,jhd->ihgd", torch.softmax(sc, dim=-1), v).reshape(i1 - i0, hq, -1)
            lse[t0 + i0:t0 + i1] = torch.logsumexp(sc, dim=-1).permute(2, 0, 1).reshape(i1 - i0, hq)
        t0 += n
    return {"out": out, "lse": lse}
