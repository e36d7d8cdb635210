"""Cases of the cross-attention and cache-eviction operators: inputs, plain forms and the library's calls.

Four operators over one paged KV pool (bf16 [pages][2][Hkv][P][D] behind a block table):

  cross    out = softmax(scale q K^T) V over the len_r cached states of request r, n_r query tokens, no causal mask
  weights  w[r, kh, j] = decay w[r, kh, j] + sum over tokens and heads of exp(scale q.k_j - lse): accumulated attention weight
  select   per (request, KV head) the positions of largest weight, some protected, ascending, ties to the lowest index
  compact  the kept K/V rows and weights moved to the head of fresh pages
"""
import math
import random

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------------------------------------------------
def _case(name, op, hq, hkv, d, page, batch, lo, hi, **more):
    c = {"op": op, "hq": hq, "hkv": hkv, "d": d, "page": page, "batch": batch, "lo": lo, "hi": hi}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # two requests, one decoder token each, short encoder outputs: nothing but launch latency
        _case("cross_decode_tiny", "cross", 4, 1, 64, 16, 2, 100, 512, q_lo=1, q_hi=1),
        # a full decode batch at the serving heads against long encoder outputs: the K/V stream
        _case("cross_decode_b64", "cross", 64, 8, 128, 64, 64, 4096, 32768, q_lo=1, q_hi=1),
        # decoder prompts of ragged lengths against encoder outputs that may be empty: the matrix products
        _case("cross_prompt_b8", "cross", 64, 8, 128, 64, 8, 0, 8192, q_lo=257, q_hi=512),
        # a few tokens per request (drafts, short prompts), odd group and page size
        _case("cross_short_prompt_g5", "cross", 20, 4, 128, 32, 16, 1, 4099, q_lo=2, q_hi=37),
        # every decode step of a batch that accumulates weights for a later eviction
        _case("weights_decode_b64", "weights", 64, 8, 128, 64, 64, 4096, 32768, q_lo=1, q_hi=1, causal=True, decay=1.0),
        # the end of a prompt: the last 64 tokens vote on what the prompt's cache keeps
        _case("weights_observe_b8", "weights", 64, 8, 128, 64, 8, 0, 16384, q_lo=33, q_hi=64, causal=True, decay=0.0),
        # cross attention's cached states, weighted by a ragged decoder prompt, small heads and pages, odd lengths
        _case("weights_cross_g4", "weights", 4, 1, 64, 16, 5, 0, 1023, q_lo=0, q_hi=301, causal=False, decay=0.9),
        # one short request: latency
        _case("select_tiny", "select", 4, 1, 64, 16, 2, 100, 512, keep=64, first=4, last=16),
        # ordinary contexts, budgets below and above the context
        _case("select_b64", "select", 64, 8, 128, 64, 64, 1024, 32768, keep=2048, first=4, last=128),
        # the longest contexts
        _case("select_b16_256k", "select", 64, 8, 128, 64, 16, 65536, 262144, keep=8191, first=4, last=128),
        # one request's eviction
        _case("compact_b1", "compact", 64, 8, 128, 64, 1, 2000, 2000, keep=777),
        # a batch's eviction
        _case("compact_b32", "compact", 64, 8, 128, 64, 32, 4096, 16384, keep=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["cross", "weights", "select", "compact"])
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 64])
    group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 8])
    hkv = rng.choice([1, 2, 3, 4, 8])
    top = 32768 if op != "select" else 262144
    hi = _log_int(rng, 48, top)
    lo = rng.choice([0, rng.randint(0, hi // 2), rng.randint(hi // 2, hi)])
    batch = _log_int(rng, 1, 64)
    more = {}
    if op in ("cross", "weights"):
        more["q_hi"] = rng.choice([1, _log_int(rng, 2, 512)])
        more["q_lo"] = more["q_hi"] if more["q_hi"] == 1 else rng.randint(0, more["q_hi"])
        # no more than the largest listed case of its kind: padded scores and cached rows
        while batch > 1 and (batch * more["q_hi"] * hi * group * hkv > 1.5e9 or batch * hi * hkv * d > 1.0e9):
            batch = max(1, batch // 2)
        while more["q_hi"] * hi * group * hkv > 1.5e9:
            hi //= 2
            lo = min(lo, hi)
    if op == "weights":
        more["causal"] = rng.random() < 0.5
        more["decay"] = rng.choice([0.0, 0.9, 1.0])
    if op == "select":
        while batch > 1 and batch * hi * hkv > 24e6:
            batch = max(1, batch // 2)
    if op == "compact":
        while batch > 1 and batch * hi * hkv * d > 0.4e9:
            batch = max(1, batch // 2)
    if op in ("select", "compact"):
        more["keep"] = _log_int(rng, 1, max(2, hi // 2))
    if op == "select":
        more["first"] = rng.choice([0, 1, 4])
        more["last"] = rng.choice([0, 1, rng.randint(0, min(128, more["keep"]))])
    return _case(None, op, group * hkv, hkv, d, page, batch, lo, hi, **more)


def _lens(case):
    """(cached length, query tokens, positions to keep) of each request: of the case alone, the same for every seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    b = case["batch"]
    ctx = [rng.randint(case["lo"], case["hi"]) for _ in range(b)]
    ctx[rng.randrange(b)] = case["hi"]
    if b > 2:
        ctx[0] = case["lo"]  # the shortest one; an empty one where the range has it
    q = [rng.randint(case.get("q_lo", 1), case.get("q_hi", 1)) for _ in range(b)]
    q[-1] = case.get("q_hi", 1)
    keep = [max(1, case.get("keep", 1) - rng.randint(0, case.get("keep", 1) // 4)) for _ in range(b)]
    keep[-1] = case.get("keep", 1)
    return ctx, q, keep


def work(case):
    ctx, q, keep = _lens(case)
    hq, hkv, d, op = case["hq"], case["hkv"], case["d"], case["op"]
    row = hkv * d * 2
    pairs = sum(n * c for n, c in zip(q, ctx))
    if op == "cross":
        return {"bytes": 2 * row * sum(c for n, c in zip(q, ctx) if n) + sum(q) * hq * (4 * d + 4), "flops": 4 * pairs * hq * d}
    if op == "weights":
        extra = 1 if case["causal"] else 0
        kv = sum(c + extra * n for n, c in zip(q, ctx))
        seen = sum(c + extra * n for n, c in zip(q, ctx) if n)
        more = sum(n * (n + 1) // 2 for n in q) if case["causal"] else 0
        return {"bytes": row * seen + kv * hkv * (4 if case["decay"] == 0.0 else 8) + sum(q) * hq * (2 * d + 4), "flops": 2 * (pairs + more) * hq * d}
    kept = sum(min(k, c) for k, c in zip(keep, ctx))
    if op == "select":
        return {"bytes": 4 * hkv * (sum(ctx) + case["batch"] * case["keep"]), "flops": sum(ctx) * hkv}
    return {"bytes": 4 * row * kept + 12 * hkv * kept, "flops": 0}


# ---------------------------------------------------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------------------------------------------------
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ctx, q_len, keep = _lens(case)
    op, b, hq, hkv, d, page = (case[k] for k in ("op", "batch", "hq", "hkv", "d", "page"))
    causal = bool(case.get("causal"))
    s = {"case": case, "ctx": _i32(ctx), "max_ctx": max(ctx), "scale": 1.0 / math.sqrt(d)}
    cached = [c + (n if causal else 0) for c, n in zip(ctx, q_len)]  # rows the cache holds by the time of the call
    if op != "select":
        # pages of a request in any order; the slots behind its last row hold what an earlier request left there
        blocks = max(1, -(-max(cached) // page))
        fresh = max(1, -(-case["keep"] // page)) if op == "compact" else 0
        used = [-(-c // page) for c in cached]
        pages = sum(used) + b * fresh + 1
        s["pool"] = torch.randn((pages, 2, hkv, page, d), generator=g, device="cuda", dtype=torch.bfloat16)
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        start = torch.tensor([sum(used[:r]) for r in range(b)], device="cuda")[:, None]
        at = torch.arange(blocks, device="cuda")[None, :]
        inside = at < torch.tensor(used, device="cuda")[:, None]
        s["table"] = torch.where(inside, perm[(start + at).clamp_(max=pages - 1)], perm[-1]).to(torch.int32).contiguous()
        if fresh:
            s["dst_table"] = perm[sum(used):sum(used) + b * fresh].reshape(b, fresh).contiguous()
    if op in ("cross", "weights"):
        total = sum(q_len)
        s["q"] = torch.randn((total, hq, d), generator=g, device="cuda", dtype=torch.bfloat16)
        s["q_len"], s["total_q"], s["max_q"] = q_len, total, max(q_len)
        s["indptr"] = _i32([sum(q_len[:r]) for r in range(b + 1)])
        # where each token sits in a batch padded to the longest request
        s["slot"] = torch.tensor([r * max(q_len) + i for r in range(b) for i in range(q_len[r])], dtype=torch.int64, device="cuda")
        s["out"] = torch.zeros((total, hq, d), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((total, hq), dtype=torch.float32, device="cuda")
    if op == "weights":
        sc, seen = _scores(s)
        s["lse"] = _unpad_rows(s, _lse(sc.masked_fill_(~seen, -math.inf))[0]).contiguous()
        del sc, seen
        stride = max(cached) + 5
        s["weights"] = torch.rand((b, hkv, stride), generator=g, device="cuda") * 0.5
    if op == "select":
        # accumulated weights: a few keys hold most of the mass, some were never attended to
        s["weights"] = torch.exp(2.0 * torch.randn((b, hkv, max(ctx) + 3), generator=g, device="cuda") - 6.0)
        s["weights"].masked_fill_(torch.rand(s["weights"].shape, generator=g, device="cuda") < 0.0625, 0.0)
    if op in ("select", "compact"):
        s["keep"] = _i32(keep)
        s["keep_idx"] = torch.zeros((b, hkv, case["keep"]), dtype=torch.int32, device="cuda")
        s["kept"] = torch.zeros((b,), dtype=torch.int32, device="cuda")
    if op == "compact":
        s["kept"] = torch.minimum(s["keep"], s["ctx"])
        order = torch.rand((b, hkv, max(ctx)), generator=g, device="cuda")
        order.masked_fill_(torch.arange(max(ctx), device="cuda") >= s["ctx"][:, None, None], 2.0)
        order = order.argsort(dim=-1)[..., : case["keep"]]
        live = torch.arange(order.shape[-1], device="cuda") < s["kept"][:, None, None]
        order = torch.where(live, order, 1 << 30).sort(dim=-1).values
        s["keep_idx"].fill_(-1)
        s["keep_idx"][..., : order.shape[-1]] = torch.where(order < (1 << 30), order, -1).to(torch.int32)
        s["weights"] = torch.rand((b, hkv, max(ctx)), generator=g, device="cuda")
        s["weights_out"] = torch.zeros((b, hkv, case["keep"]), dtype=torch.float32, device="cuda")
    if own:
        _open(s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------------------------------------------------
_handles = {}


def _open(s):
    """The handle, layer, batch and workspace that a user's program keeps."""
    from paper_2607_13095_b200 import binding as hb
    c = s["case"]
    key = (c["hq"], c["hkv"], c["d"], c["page"])
    if key not in _handles:
        _handles[key] = hb.Handle(*key, out_dtype=torch.bfloat16)
    s["hb"], s["h"] = hb, _handles[key]
    if "pool" in s:
        s["layer"] = hb.Layer(s["pool"], False)
        ring = torch.zeros((c["batch"], s["h"].ring_pages), dtype=torch.int32, device="cuda")
        head = torch.zeros((c["batch"],), dtype=torch.int32, device="cuda")
        one = c.get("q_lo", 1) == 1 and c.get("q_hi", 1) == 1
        s["batch"] = hb.Batch(s["ctx"], s["table"], ring, head, None if one else s["indptr"], max_q_len=s.get("max_q", 1),
                              total_q=s.get("total_q", c["batch"]), max_ctx_len=s["max_ctx"])
    if c["op"] == "cross":
        need = hb.hswa_cross_workspace_need(s["h"], c["batch"], s["total_q"], s["max_q"], s["max_ctx"])
        s["ws"] = torch.empty((max(need, 256),), dtype=torch.uint8, device="cuda")


def _run_own(s):
    hb, c = s["hb"], s["case"]
    if c["op"] == "cross":
        hb.hswa_cross_attn(s["h"], s["layer"], s["batch"], s["q"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "weights":
        hb.hswa_attn_weights(s["h"], s["layer"], s["batch"], c["causal"], s["q"], s["lse"], c["decay"], s["weights"])
        return {"weights": s["weights"]}
    if c["op"] == "select":
        hb.hswa_evict_select(s["h"], c["batch"], s["ctx"], s["max_ctx"], s["weights"], s["keep"], s["keep_idx"], s["kept"],
                             protect_first=c["first"], protect_last=c["last"])
        return {"keep_idx": s["keep_idx"], "kept": s["kept"]}
    hb.hswa_evict_compact(s["h"], s["layer"], s["batch"], s["keep_idx"], s["kept"], s["dst_table"], s["weights"], s["weights_out"])
    return {"pool": s["pool"], "weights": s["weights_out"]}


# ---------------------------------------------------------------------------------------------------------------------
# Plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _gather(s, which):
    """The cached K (0) or V (1) of every request, padded: [B][Hkv][L][D] in 32 bits."""
    t = s["pool"][s["table"].long(), which]  # [B][blocks][Hkv][P][D]
    b, n, h, p, d = t.shape
    return t.permute(0, 2, 1, 3, 4).reshape(b, h, n * p, d).float()


def _pad_rows(s, x):
    """[T][Hq][...] -> [B][Hkv][tokens * G][...], padded to the longest request."""
    c = s["case"]
    rest = x.shape[2:]
    y = torch.zeros((c["batch"] * s["max_q"], *x.shape[1:]), dtype=torch.float32, device=x.device)
    y[s["slot"]] = x.float()
    g = c["hq"] // c["hkv"]
    return y.reshape(c["batch"], s["max_q"], c["hkv"], g, *rest).transpose(1, 2).reshape(c["batch"], c["hkv"], s["max_q"] * g, *rest)


def _unpad_rows(s, y):
    c = s["case"]
    rest = y.shape[3:]
    g = c["hq"] // c["hkv"]
    y = y.reshape(c["batch"], c["hkv"], s["max_q"], g, *rest).transpose(1, 2).reshape(c["batch"] * s["max_q"], c["hq"], *rest)
    return y[s["slot"]]


def _scores(s):
    """Scaled scores [B][Hkv][tokens * G][L] and which keys each row sees."""
    c = s["case"]
    k = _gather(s, 0)
    sc = (_pad_rows(s, s["q"]) * s["scale"]) @ k.transpose(2, 3)
    j = torch.arange(k.shape[2], device=k.device)
    if c.get("causal"):
        token = torch.arange(s["max_q"], device=k.device).repeat_interleave(c["hq"] // c["hkv"])
        seen = j[None, None, :] <= s["ctx"][:, None, None] + token[None, :, None]
    else:
        seen = (j[None, :] < s["ctx"][:, None])[:, None, :]
    return sc, seen[:, None]


def _lse(sc):
    m = sc.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(sc - m)
    total = e.sum(dim=-1, keepdim=True)
    return (m + torch.log(total))[..., 0], e, total


def _plain_cross(s):
    sc, seen = _scores(s)
    lse, e, total = _lse(sc.masked_fill_(~seen, -math.inf))
    del sc
    out = torch.where(total > 0, (e @ _gather(s, 1)) / total, 0.0)
    return {"out": _unpad_rows(s, out).to(torch.bfloat16), "lse": _unpad_rows(s, lse).contiguous()}


def _plain_weights(s):
    c = s["case"]
    sc, seen = _scores(s)
    lse = _pad_rows(s, s["lse"])[..., None]
    valid = torch.zeros((c["batch"] * s["max_q"], c["hq"]), device=sc.device)
    valid[s["slot"]] = 1.0
    g = c["hq"] // c["hkv"]
    valid = valid.reshape(c["batch"], s["max_q"], c["hkv"], g).transpose(1, 2).reshape(c["batch"], c["hkv"], -1, 1) > 0
    w = torch.where(seen & valid & (lse > -math.inf), torch.exp(sc.sub_(lse)), 0.0).sum(dim=2)
    del sc
    # positions the cache held before the step keep what they had, those of this step start at nothing
    buf = s["weights"]
    w = torch.nn.functional.pad(w, (0, max(0, buf.shape[2] - w.shape[2])))[..., : buf.shape[2]]
    j = torch.arange(buf.shape[2], device=buf.device)[None, None, :]
    ctx = s["ctx"][:, None, None]
    new = torch.tensor(s["q_len"], device=buf.device)[:, None, None] if c["causal"] else 0
    before = torch.where(j < ctx, buf, 0.0) * c["decay"] if c["decay"] else torch.zeros_like(buf)
    buf.copy_(torch.where(j < ctx + new, before + w, buf))
    return {"weights": buf}


def _plain_select(s):
    c = s["case"]
    w = s["weights"][..., : s["max_ctx"]]
    j = torch.arange(w.shape[-1], device=w.device)
    ctx = s["ctx"][:, None, None]
    rank = torch.where((j < c["first"]) | (j >= ctx - c["last"]), math.inf, w).masked_fill_(j >= ctx, -math.inf)
    kept = torch.minimum(s["keep"], s["ctx"])
    order = rank.sort(dim=-1, descending=True, stable=True).indices[..., : c["keep"]]
    live = torch.arange(order.shape[-1], device=w.device) < kept[:, None, None]
    order = torch.where(live, order, 1 << 30).sort(dim=-1).values
    s["keep_idx"].fill_(-1)
    s["keep_idx"][..., : order.shape[-1]] = torch.where(order < (1 << 30), order, -1).to(torch.int32)
    s["kept"].copy_(kept)
    return {"keep_idx": s["keep_idx"], "kept": s["kept"]}


def _plain_compact(s):
    c, pool = s["case"], s["pool"]
    live = s["keep_idx"] >= 0
    src = s["keep_idx"].clamp(min=0).long()
    r = torch.arange(c["batch"], device=src.device)[:, None, None]
    kh = torch.arange(c["hkv"], device=src.device)[None, :, None]
    i = torch.arange(c["keep"], device=src.device)[None, None, :]
    page, slot = s["table"][r, src // c["page"]].long(), src % c["page"]
    to_page, to_slot = s["dst_table"][r, i // c["page"]].long(), i % c["page"]
    # places behind the last kept row get what they hold already
    pool[to_page, :, kh, to_slot] = torch.where(live[..., None, None], pool[page, :, kh, slot], pool[to_page, :, kh, to_slot])
    s["weights_out"].copy_(torch.where(live, s["weights"].gather(2, src), s["weights_out"]))
    return {"pool": s["pool"], "weights": s["weights_out"]}


def run(state):
    if own:
        return _run_own(state)
    return {"cross": _plain_cross, "weights": _plain_weights, "select": _plain_select, "compact": _plain_compact}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits, request by request
# ---------------------------------------------------------------------------------------------------------------------
def _rows(s, r, n):
    """K and V of request r's first n cached positions, [n][Hkv][D] in 64 bits."""
    page = s["case"]["page"]
    pos = torch.arange(n, device="cuda")
    pages = s["table"][r].long()[pos // page]
    both = s["pool"][pages, :, :, pos % page].double()  # [n][2][Hkv][D]
    return both[:, 0], both[:, 1]


def exact(case, seed):
    if case["op"] == "select":
        return None
    s = prepare(case, seed)
    hq, hkv = case["hq"], case["hkv"]
    g = hq // hkv
    ctx, q_len, _ = _lens(case)
    if case["op"] == "compact":
        pool, w_out = s["pool"].clone(), s["weights_out"].double()
        for r in range(case["batch"]):
            n = int(s["kept"][r])
            for kh in range(hkv):
                src = s["keep_idx"][r, kh, :n].long()
                dst = torch.arange(n, device="cuda")
                rows = s["pool"][s["table"][r].long()[src // case["page"]], :, kh, src % case["page"]]
                pool[s["dst_table"][r].long()[dst // case["page"]], :, kh, dst % case["page"]] = rows
                w_out[r, kh, :n] = s["weights"][r, kh, src].double()
        return {"pool": pool, "weights": w_out}
    out = torch.zeros((sum(q_len), hq, case["d"]), dtype=torch.float64, device="cuda")
    lse = torch.full((sum(q_len), hq), -math.inf, dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if case["op"] == "weights" else None
    t0 = 0
    for r in range(case["batch"]):
        c, n = ctx[r], q_len[r]
        total = c + n if case.get("causal") else c
        k, v = _rows(s, r, total)
        if weights is not None:
            old = weights[r, :, :c] * case["decay"] if case["decay"] else torch.zeros_like(weights[r, :, :c])
            weights[r, :, :c] = old
            weights[r, :, c:total] = 0.0
        step = max(1, int(1e8 // max(1, total * hq)))
        for i0 in range(0, n if total else 0, step):
            i1 = min(n, i0 + step)
            q = s["q"][t0 + i0:t0 + i1].double().reshape(i1 - i0, hkv, g, -1)
            sc = torch.einsum("ihgd,jhd->hgij", q, k) / math.sqrt(case["d"])
            if case.get("causal"):
                late = torch.arange(total, device="cuda")[None, :] > c + torch.arange(i0, i1, device="cuda")[:, None]
                sc = sc.masked_fill(late, -math.inf)
            if weights is not None:
                given = s["lse"][t0 + i0:t0 + i1].double().reshape(i1 - i0, hkv, g).permute(1, 2, 0)[..., None]
                weights[r, :, :total] += torch.where(given > -math.inf, torch.exp(sc - given), 0.0).sum(dim=(1, 2))
            else:
                p = torch.softmax(sc, dim=-1)
                out[t0 + i0:t0 + i1] = torch.einsum("hgij,jhd->ihgd", p, v).reshape(i1 - i0, hq, -1)
                lse[t0 + i0:t0 + i1] = torch.logsumexp(sc, dim=-1).permute(2, 0, 1).reshape(i1 - i0, hq)
        t0 += n
    return {"weights": weights} if weights is not None else {"out": out, "lse": lse}
