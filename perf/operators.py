"""What is timed of the operators on a context cache: attention that reads part
of it, a cache held in 4 bits, and eviction from it.

A case is a dict of plain values.  Its `kind` says which public entry points a
pass goes through:

  attn     attention of a draft block (`tree` false) or of a verified tree over
           a context cache, dense or in 4 bits (`format`), the whole of it or
           the last `window` positions and the first `sinks` ones (window 0: all)
  convert  a dense cache into a 4-bit one, and that one back into a dense one
  weigh    attention weight accumulated per cache slot from a call's queries and
           log-sum-exps: of all rows of a block, or of the rows of an accepted
           path (`path`)
  evict    the `budget` slots of each sequence and KV head that are kept,
           compacted in order into another cache

`own` chooses between the library's kernels and the same mathematics in
elementary torch operations.  Context lengths of a ragged batch are spread
between `ctx_lo` and `ctx` by the golden ratio, so that the work of a case does
not depend on the seed; all values, trees and paths do.
"""

import math
import random

import torch

own = False

PATH_STRIDE = 16  # holds any accepted path of a tree of depth <= 15
DEPTH_CAP = 15    # offsets of a 16-row draft block
BLOCK = 32        # values of a 4-bit cache that share a scale
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    qwen = {"hq": 28, "hkv": 4, "d": 128, "dtype": "bf16"}
    full = {"window": 0, "sinks": 0}
    return [
        # the smallest call: the tiny fp32 decoder on which losslessness is
        # audited, its tree verified within a short window; latency
        {"name": "window verify tiny fp32", "kind": "attn", "tree": True, "format": "dense", "batch": 1, "ctx": 256, "ctx_lo": 256,
         "hq": 4, "hkv": 1, "d": 64, "dtype": "f32", "n": 16, "window": 64, "sinks": 4, "lse": True},
        # plain decoding, one token a sequence, of sixteen ragged conversations
        # whose layer attends to a window
        {"name": "window step x16", "kind": "attn", "tree": False, "format": "dense", "batch": 16, "ctx": 32768, "ctx_lo": 2048,
         "n": 1, "window": 4096, "sinks": 4, "lse": False, **qwen},
        # the tree of a long document, verified within a window
        {"name": "window verify 16k x4", "kind": "attn", "tree": True, "format": "dense", "batch": 4, "ctx": 16384, "ctx_lo": 16384,
         "n": 64, "window": 4096, "sinks": 64, "lse": False, **qwen},
        # interactive use, one token of one sequence over a 4-bit cache
        {"name": "kv4 step 4k x1", "kind": "attn", "tree": False, "format": "kv4", "batch": 1, "ctx": 4096, "ctx_lo": 4096,
         "n": 1, "lse": False, **full, **qwen},
        # a draft block over a long document's 4-bit cache
        {"name": "kv4 draft 16k x4", "kind": "attn", "tree": False, "format": "kv4", "batch": 4, "ctx": 16384, "ctx_lo": 16384,
         "n": 16, "lse": False, **full, **qwen},
        # the largest: a ragged batch's trees over 4-bit caches
        {"name": "kv4 verify ragged x16", "kind": "attn", "tree": True, "format": "kv4", "batch": 16, "ctx": 32768, "ctx_lo": 2048,
         "n": 64, "lse": False, **full, **qwen},
        # both at once, in fp32, with odd sizes
        {"name": "kv4 window verify fp32 d64 x3", "kind": "attn", "tree": True, "format": "kv4", "batch": 3, "ctx": 11003, "ctx_lo": 1037,
         "hq": 8, "hkv": 2, "d": 64, "dtype": "f32", "n": 37, "window": 2500, "sinks": 5, "lse": True},
        # a prefilled cache goes into 4 bits, and a 4-bit one back
        {"name": "kv4 convert 16k x4", "kind": "convert", "batch": 4, "ctx": 16384, "ctx_lo": 16384, "hkv": 4, "d": 128, "dtype": "bf16"},
        # a verified round's weights: the rows of the accepted path
        {"name": "weigh path 16k x4", "kind": "weigh", "format": "dense", "path": True, "batch": 4, "ctx": 16384, "ctx_lo": 16384,
         "n": 64, "decay": 1.0, **full, **qwen},
        # a draft block's weights over ragged 4-bit caches, old ones fading
        {"name": "weigh kv4 block ragged x16", "kind": "weigh", "format": "kv4", "path": False, "batch": 16, "ctx": 32768, "ctx_lo": 2048,
         "n": 16, "decay": 0.9, **full, **qwen},
        # a long document's cache cut to a quarter
        {"name": "evict 16k to 4k x4", "kind": "evict", "batch": 4, "ctx": 16384, "ctx_lo": 16384, "hkv": 4, "d": 128, "dtype": "bf16",
         "budget": 4096, "sinks": 4, "recent": 512},
        # a ragged batch's, some of which fit the budget as they are
        {"name": "evict ragged f32 d64 x5", "kind": "evict", "batch": 5, "ctx": 11003, "ctx_lo": 1037, "hkv": 2, "d": 64, "dtype": "f32",
         "budget": 5001, "sinks": 5, "recent": 301},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """The same four kinds over the ranges the listed cases span: one token to 64
    rows, 1 to 16 sequences, short to 32k contexts, odd sizes among them, both
    head sizes and types.  fp32 attention is drawn smaller (its matrix rate is a
    ninth)."""
    kind = rng.choice(("attn", "attn", "attn", "convert", "weigh", "evict"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    small = dtype == "f32" and kind in ("attn", "weigh")
    hq, hkv = rng.choice(((28, 4), (8, 2), (4, 1), (6, 3), (16, 16), (12, 1)))
    d = rng.choice((64, 128))
    batch = _log_int(rng, 1, 4 if small else 16)
    ctx = _log_int(rng, 48, 8192 if small else 32768)
    case = {"kind": kind, "batch": batch, "ctx": ctx, "ctx_lo": rng.choice((ctx, max(1, ctx // 13))), "hkv": hkv, "d": d, "dtype": dtype}
    if kind in ("attn", "weigh"):
        window = rng.choice((0, _log_int(rng, 16, max(17, ctx))))
        case.update(hq=hq, n=rng.choice((1, 2, 16, 64, rng.randint(3, 63))), format=rng.choice(("dense", "kv4")),
                    window=window, sinks=rng.randint(0, 80) if window else 0)
    if kind == "attn":
        case.update(tree=rng.random() < 0.6, lse=dtype == "f32")
        if not window and case["format"] == "dense":
            case.update(window=_log_int(rng, 16, max(17, ctx)), sinks=rng.randint(0, 80))
    elif kind == "weigh":
        case.update(path=rng.random() < 0.5, decay=rng.choice((0.0, 0.9, 1.0)))
    elif kind == "evict":
        budget = _log_int(rng, max(1, ctx // 16), ctx)
        sinks = min(rng.randint(0, 80), budget // 4)
        case.update(budget=budget, sinks=sinks, recent=rng.randint(0, budget // 3))
    return case


# ---------------------------------------------------------------- inputs
def _lens(case):
    lo, hi, n = case["ctx_lo"], case["ctx"], case["batch"]
    if lo == hi:
        return [hi] * n
    lens = [lo + int((hi - lo) * ((0.6180339887 * (i + 1)) % 1.0)) for i in range(n)]
    lens[-1] = hi
    return lens


def _tree(n, rng):
    """Parents of a tree with a deep spine and side branches, and a path in it
    from the root."""
    parents, depth = [-1], [0]
    for c in range(1, n):
        v = rng.randrange(max(0, c - 4), c)
        while depth[v] >= DEPTH_CAP:
            v = parents[v]
        parents.append(v)
        depth.append(depth[v] + 1)
    path, v = [], rng.randrange(n)
    while v >= 0:
        path.append(v)
        v = parents[v]
    return parents, path[::-1]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _quantise(x):
    """Codes and scale bytes of [..., d] values: 32 in a row share 2^e with e two
    below the exponent of their largest magnitude (of the next power of two from
    1.75 times a power on), each is the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6
    times 2^e, ties to the even code, at most 6."""
    y = x.float().unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(y.abs().amax(-1))  # largest = m 2^e, m in [0.5, 1)
    e = torch.where(m > 0, e - 3 + (m >= 0.875).int(), -125).clamp(min=-125)
    a = (y.double() * torch.exp2(-e.double()).unsqueeze(-1)).abs()
    q = torch.where(a < 2, torch.round(a * 2), torch.where(a < 4, torch.round(a) + 2, torch.round(a / 2) + 4)).clamp(max=7)
    code = (q + 8 * torch.signbit(y)).to(torch.uint8).flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] | code[..., 1] << 4, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What a 4-bit cache's codes and scales stand for, in 32 bits."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    grid = torch.cat([grid, -grid])
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    return (grid[both].unflatten(-1, (-1, BLOCK)) * torch.exp2(scales.float() - 127).unsqueeze(-1)).flatten(-2)


def _keys(s, name):
    """The cache's keys or values in 32 bits."""
    return _values(s[name], s[name + "_scale"]) if s["format"] == "kv4" else s[name].float()


def _inputs(case, seed):
    rng = random.Random(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    b, hkv, d, cap = case["batch"], case["hkv"], case["d"], case["ctx"]
    lens = _lens(case)
    s = {"case": case, "kind": kind, "lens": _ints(lens), "format": case.get("format", "dense")}

    def normal(*shape):
        return torch.randn(shape, generator=gen, dtype=dt, device="cuda")

    # keys have some channels a few times larger than others, as a cache's have
    loud = torch.exp(0.5 * torch.randn((1, hkv, 1, d), generator=gen, device="cuda")).to(dt)
    s["k"] = normal(b, hkv, cap, d).mul_(loud)
    s["v"] = normal(b, hkv, cap, d)
    if s["format"] == "kv4":
        s["k"], s["k_scale"] = _quantise(s["k"])
        s["v"], s["v_scale"] = _quantise(s["v"])
    if kind in ("attn", "weigh"):
        n = case["n"]
        s["q"] = normal(b, n, case["hq"], d)
        s["k_new"], s["v_new"] = normal(b, n, hkv, d) * loud.squeeze(2).unsqueeze(1), normal(b, n, hkv, d)
        trees = [_tree(n, rng) for _ in range(b)]
        s["parents"] = _ints([t[0] for t in trees])
        s["path_rows"] = [t[1] for t in trees]
    if kind == "weigh":
        rows = (6 if case["path"] else n) * case["hq"] // hkv  # what eight such calls leave in a slot
        s["weights"] = torch.rand((b, hkv, cap + PATH_STRIDE), generator=gen, device="cuda") * (8.0 * rows / cap)
        s["accept_len"] = _ints([len(t) - 1 for t in s["path_rows"]])
        s["accept_path"] = _ints([t + [-1] * (PATH_STRIDE - len(t)) for t in s["path_rows"]])
        tree = dict(case, tree=case["path"])
        s["lse"] = torch.logsumexp(_scores(s, tree), -1).unflatten(-1, (n, -1)).permute(0, 2, 1, 3).flatten(2).contiguous()
    if kind == "evict":
        # accumulated weights spread over decades; some slots were never seen
        w = torch.exp(2.5 * torch.randn((b, hkv, cap), generator=gen, device="cuda") - 6)
        s["weights"] = torch.where(torch.rand(w.shape, generator=gen, device="cuda") < 0.1, 0.0, w)
        cut = case["budget"]
        s["out"] = {"k": torch.zeros((b, hkv, cut, d), dtype=dt, device="cuda"), "v": torch.zeros((b, hkv, cut, d), dtype=dt, device="cuda"),
                    "weights": torch.zeros((b, hkv, cut), device="cuda")}
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _hold(s)
    return s


def _hold(s):
    """The cache objects, outputs, workspaces and prepared calls that a serving loop keeps."""
    import paper_2609_00355_amd as G
    case, kind = s["case"], s["kind"]
    b, hkv, cap, d = case["batch"], case["hkv"], case["ctx"], case["d"]
    reach = {"n_sinks": case.get("sinks", 0), "window": case.get("window", 0)}
    if kind == "attn":
        cache = G.ContextCache(s["k"], s["v"], s["lens"], k_scale=s.get("k_scale"), v_scale=s.get("v_scale"))
        lse = torch.empty(s["q"].shape[:3], device="cuda") if case["lse"] else None
        if case["tree"]:
            s["call"], s["got"], _ = G.prepare_cache_tree_verify_attn(s["q"], cache, s["k_new"], s["v_new"], s["parents"], lse=lse, **reach)
        else:
            s["call"], s["got"], _ = G.prepare_cache_block_draft_attn(s["q"], cache, s["k_new"], s["v_new"], lse=lse, **reach)
        s["got_lse"] = lse
    elif kind == "convert":
        dense = G.ContextCache(s["k"], s["v"], s["lens"])
        packed = G.new_cache(b, hkv, cap, d, fmt="kv4")
        s["back"] = G.new_cache(b, hkv, cap, d, dtype=DTYPES[case["dtype"]])
        s["pack"], s["unpack"] = G.prepare_cache_convert(dense, packed), G.prepare_cache_convert(packed, s["back"])
    elif kind == "weigh":
        cap += PATH_STRIDE  # room for the rows that the round commits
        cache = G.new_cache(b, hkv, cap, d, dtype=DTYPES[case["dtype"]], fmt=s["format"])
        for name in ("k", "v") + (("k_scale", "v_scale") if s["format"] == "kv4" else ()):
            getattr(cache, name)[:, :, :case["ctx"]] = s[name]
        cache.ctx_lens, cache.weights = s["lens"], s["weights"]
        s["got"] = s["weights"].clone()  # slots that the call leaves alone
        path = {"k_new": s["k_new"], "accept_len": s["accept_len"], "accept_path": s["accept_path"]} if case["path"] else {}
        s["call"] = G.prepare_cache_weigh(s["q"], cache, s["lse"], decay=case["decay"], weights_out=s["got"], **path, **reach)
    else:
        src = G.ContextCache(s["k"], s["v"], s["lens"], weights=s["weights"])
        s["to"] = G.ContextCache(s["out"]["k"], s["out"]["v"], torch.zeros_like(s["lens"]), weights=s["out"]["weights"])
        s["call"], s["kept"] = G.prepare_cache_evict(src, s["to"], case["budget"], n_sinks=case["sinks"], n_recent=case["recent"])


# ---------------------------------------------------------------- plain forms
def _relations(s, tree):
    """Which new rows are a row's ancestors (itself among them), and the rows' depths."""
    n = s["q"].shape[1]
    if not tree:
        return torch.ones((1, n, n), dtype=torch.bool, device="cuda"), torch.arange(n, device="cuda").expand(s["q"].shape[0], n)
    up = torch.nn.functional.one_hot(s["parents"].long().clamp(min=0), n).double()
    up[:, 0] = 0.0
    anc = torch.linalg.matrix_power(up + torch.eye(n, device="cuda", dtype=torch.float64), n) > 0.5
    return anc, anc.sum(-1) - 1


def _scores(s, case):
    """Scaled scores [b, hkv, n * group, cap + n], -inf where a row does not see a key."""
    q, k = s["q"].float(), _keys(s, "k")
    b, n, hq, d = q.shape
    hkv, cap = k.shape[1], k.shape[2]
    q = q.unflatten(2, (hkv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    new = s["k_new"].float().transpose(1, 2)
    z = torch.cat([q @ k.transpose(-1, -2), q @ new.transpose(-1, -2)], -1) / math.sqrt(d)
    anc, depth = _relations(s, case["tree"])
    j = torch.arange(cap, device="cuda")
    ctx, at = s["lens"][:, None, None], (s["lens"][:, None] + depth)[:, :, None]
    sees, kin = (j < ctx).expand(b, n, cap), anc.expand(b, n, n)
    if case["window"]:
        sees = sees & ((j < case["sinks"]) | (j > at - case["window"]))
        if case["tree"]:
            kin = kin & ((depth[:, :, None] - depth[:, None, :] < case["window"]) | (ctx + depth[:, None, :] < case["sinks"]))
    sees = torch.cat([sees, kin], -1).repeat_interleave(hq // hkv, 1).unsqueeze(1)
    return torch.where(sees, z, -math.inf)


def _plain_attention(s):
    case = s["case"]
    z = _scores(s, case)
    n = case["n"]
    top = z.amax(-1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(-1, keepdim=True)
    v = torch.cat([_keys(s, "v"), s["v_new"].float().transpose(1, 2)], 2)
    out = (e @ v / total).unflatten(2, (n, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3).to(s["q"].dtype)
    if not case["lse"]:
        return {"out": out}
    return {"out": out, "lse": (top + torch.log(total)).squeeze(-1).unflatten(-1, (n, -1)).permute(0, 2, 1, 3).flatten(2)}


def _plain_weigh(s):
    case = s["case"]
    cap, n = case["ctx"], case["n"]
    p = torch.exp(_scores(s, dict(case, tree=case["path"])) - s["lse"].unflatten(2, (case["hkv"], -1)).permute(0, 2, 1, 3).flatten(2)[..., None])
    got = s["weights"].clone()
    j = torch.arange(got.shape[-1], device="cuda")
    ctx = s["lens"][:, None, None]
    if not case["path"]:
        return {"weights": torch.where(j < ctx, case["decay"] * got + torch.nn.functional.pad(p[..., :cap].sum(2), (0, PATH_STRIDE)), got)}
    # the rows on the path; the keys on it take the slots after the context
    t = torch.arange(PATH_STRIDE, device="cuda")
    valid = t <= s["accept_len"][:, None]
    on = torch.zeros((case["batch"], n), device="cuda").scatter_add(1, s["accept_path"].long().clamp(min=0), valid.float())
    sums = (p * on.repeat_interleave(p.shape[2] // n, 1)[:, None, :, None]).sum(2)
    got = torch.where(j < ctx, case["decay"] * got + torch.nn.functional.pad(sums[..., :cap], (0, PATH_STRIDE)), got)
    mine = torch.gather(sums[..., cap:], 2, s["accept_path"].long().clamp(min=0)[:, None].expand(-1, case["hkv"], -1))
    new = (j - ctx).clamp(0, PATH_STRIDE - 1).expand(got.shape)
    take = (j >= ctx) & (j <= ctx + s["accept_len"][:, None, None])
    return {"weights": torch.where(take, torch.gather(mine, 2, new), got)}


def _plain_evict(s):
    case, w = s["case"], s["weights"]
    budget, cap = case["budget"], w.shape[-1]
    j = torch.arange(cap, device="cuda")
    ctx = s["lens"][:, None, None]
    key = torch.where((j < case["sinks"]) | (j >= ctx - case["recent"]), math.inf, w)
    key = torch.where(j < ctx, key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :budget]
    slot = torch.sort(torch.where(order < ctx, order, cap), -1).values
    there = slot < cap
    at = slot.clamp(max=cap - 1)
    rows = at[..., None].expand(-1, -1, -1, case["d"])
    new = {name: torch.where(there[..., None], torch.gather(s[name], 2, rows), s["out"][name]) for name in ("k", "v")}
    return {**new, "weights": torch.where(there, torch.gather(w, 2, at), s["out"]["weights"]),
            "kept": torch.where(there, at, -1).int(), "lens": s["lens"].clamp(max=budget)}


def run(s):
    kind = s["kind"]
    if own:
        if kind == "convert":
            s["pack"]()
            s["unpack"]()
            return {"k": s["back"].k, "v": s["back"].v}
        s["call"]()
        if kind == "attn":
            return {"out": s["got"], "lse": s["got_lse"]} if s["case"]["lse"] else {"out": s["got"]}
        if kind == "weigh":
            return {"weights": s["got"]}
        to = s["to"]
        return {"k": to.k, "v": to.v, "weights": to.weights, "kept": s["kept"], "lens": to.ctx_lens}
    if kind == "attn":
        return _plain_attention(s)
    if kind == "weigh":
        return _plain_weigh(s)
    if kind == "evict":
        return _plain_evict(s)
    # slots past a sequence's length are no part of either cache
    live = (torch.arange(s["k"].shape[2], device="cuda") < s["lens"][:, None])[:, None, :, None]
    return {name: torch.where(live, _values(*_quantise(s[name])), 0.0).to(s[name].dtype) for name in ("k", "v")}


# ---------------------------------------------------------------- work
def work(case):
    """Inputs read once, outputs written once, and the matrix products.  A
    windowed call cannot do without the keys that some row sees, each 4-bit key
    or value is d / 2 bytes of codes and d / 32 of scales, and the weights need
    the keys alone."""
    kind, lens = case["kind"], _lens(case)
    b, hkv, d = case["batch"], case["hkv"], case["d"]
    esz = 4 if case["dtype"] == "f32" else 2
    row = d / 2 + d / BLOCK if case.get("format") == "kv4" else d * esz
    if kind == "convert":
        return {"bytes": 2.0 * sum(lens) * hkv * (2 * d * esz + d / 2 + d / BLOCK) + 4 * b, "flops": 0.0}
    if kind == "evict":
        kept = sum(min(x, case["budget"]) for x in lens)
        read = sum(x for x in lens if x > case["budget"]) * hkv * 4.0
        return {"bytes": read + kept * hkv * (4 * d * esz + 12.0) + 8 * b, "flops": 0.0}
    n, hq, w = case["n"], case["hq"], case["window"]
    seen = [min(x, min(case["sinks"], x) + w - 1) if w else x for x in lens]
    if kind == "attn":
        nbytes = 2.0 * sum(seen) * hkv * row + (2 * hq + 2 * hkv) * b * n * d * esz + 4 * b + (4 * b * n * hq if case["lse"] else 0)
        return {"bytes": nbytes, "flops": 4.0 * d * hq * n * (sum(seen) + b * n / 4)}
    rows = 6 if case["path"] else n  # a path has about six rows
    old = 2 if case["decay"] else 1
    nbytes = sum(seen) * hkv * row + 4.0 * old * sum(lens) * hkv + b * rows * hq * (d * esz + 4.0)
    return {"bytes": nbytes, "flops": 2.0 * d * hq * rows * sum(seen)}


# ---------------------------------------------------------------- in 64 bits
def _exact_values(s, name):
    if s["format"] != "kv4":
        return s[name].double()
    codes = s[name].short()
    out = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = codes >> 4 * half & 15
        e, m = c >> 1 & 3, (c & 1).double()  # one sign, two exponent and one fraction bit
        a = torch.where(e == 0, m / 2, (1 + m / 2) * torch.pow(2.0, (e - 1).double()))
        out[..., half::2] = torch.where(c > 7, -a, a)
    return out * torch.pow(2.0, s[name + "_scale"].double() - 127).repeat_interleave(BLOCK, -1)


def _exact_rows(s, case, i, tree):
    """One sequence's scores [hkv][rows of (new row, query head)][ctx + n] in 64
    bits and the new rows' depths."""
    ctx, n, hkv = _lens(case)[i], case["n"], case["hkv"]
    group = case["hq"] // hkv
    k = torch.cat([_exact_values({"format": s["format"], "k": s["k"][i], "k_scale": s["k_scale"][i] if "k_scale" in s else None}, "k")[:, :ctx],
                   s["k_new"][i].double().transpose(0, 1)], 1)
    q = s["q"][i].double().reshape(n, hkv, group, -1).transpose(0, 1).reshape(hkv, n * group, -1)
    z = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(case["d"])
    parents = s["parents"][i].tolist()
    depth, sees = list(range(n)), torch.ones((n, n), dtype=torch.bool)
    if tree:
        sees = torch.eye(n, dtype=torch.bool)
        depth[0] = 0
        for v in range(1, n):
            sees[v] |= sees[parents[v]]
            depth[v] = depth[parents[v]] + 1
    whole = torch.ones((n, ctx + n), dtype=torch.bool)
    whole[:, ctx:] = sees
    for v in range(n):
        if case["window"]:
            whole[v, min(ctx, case["sinks"]):max(min(ctx, case["sinks"]), min(ctx, ctx + depth[v] - case["window"] + 1))] = False
            for u in range(n if tree else 0):
                if depth[v] - depth[u] >= case["window"] and ctx + depth[u] >= case["sinks"]:
                    whole[v, ctx + u] = False
    return z.masked_fill(~whole.repeat_interleave(group, 0).to(z.device), -math.inf)


def exact(case, seed):
    s = _inputs(case, seed)
    kind, lens = case["kind"], _lens(case)
    b, hkv, d = case["batch"], case["hkv"], case["d"]
    if kind == "convert":
        got = {}
        for name in ("k", "v"):
            x = s[name].double().reshape(b, hkv, -1, d // BLOCK, BLOCK)
            top = x.abs().amax(-1, keepdim=True)
            power = torch.floor(torch.log2(top.clamp(min=1e-300)))
            power = torch.where(top >= 1.75 * torch.pow(2.0, power), power + 1, power) - 2
            unit = torch.pow(2.0, power.clamp(min=-125))
            grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
            a = x.abs() / unit
            mid = (grid[1:] + grid[:-1]) / 2
            up = torch.bucketize(a, mid, right=True)      # a border goes up
            down = torch.bucketize(a, mid, right=False)   # a border stays below
            code = torch.where(up % 2 == 0, up, down)     # the even one of the two
            y = (grid[code] * unit * torch.sign(x)).reshape(b, hkv, -1, d)
            for i, n in enumerate(lens):
                y[i, :, n:] = 0.0
            got[name] = y
        return got
    if kind == "evict":
        budget, names = case["budget"], ("k", "v", "weights")
        got = {name: s["out"][name].double() for name in names}
        for i, n in enumerate(lens):
            for g in range(hkv):
                w = s["weights"][i, g, :n].tolist()
                mid = range(min(case["sinks"], n), max(min(case["sinks"], n), n - case["recent"]))
                best = sorted(mid, key=lambda x: (-w[x], x))[:budget - (n - len(mid))] if n > budget else mid
                kept = sorted(set(range(n)) - set(mid) | set(best))
                for name in names:
                    got[name][i, g, :len(kept)] = s[name][i, g, kept].double()
        return {**got, "kept": None, "lens": None}
    if kind == "attn":
        n, hq = case["n"], case["hq"]
        out = torch.empty((b, n, hq, d), dtype=torch.float64, device="cuda")
        lse = torch.empty((b, n, hq), dtype=torch.float64, device="cuda")
        for i in range(b):
            z = _exact_rows(s, case, i, case["tree"])
            total = torch.logsumexp(z, -1, keepdim=True)
            v = torch.cat([_exact_values({"format": s["format"], "v": s["v"][i], "v_scale": s["v_scale"][i] if "v_scale" in s else None}, "v")[:, :lens[i]],
                           s["v_new"][i].double().transpose(0, 1)], 1)
            o = torch.matmul(torch.exp(z - total), v)
            out[i] = o.reshape(hkv, n, -1, d).transpose(0, 1).reshape(n, hq, d)
            lse[i] = total.reshape(hkv, n, -1).transpose(0, 1).reshape(n, hq)
        return {"out": out, "lse": lse} if case["lse"] else {"out": out}
    got = s["weights"].double()
    group = case["hq"] // hkv
    for i, ctx in enumerate(lens):
        lse = s["lse"][i].double().reshape(case["n"], hkv, group).transpose(0, 1)
        p = torch.exp(_exact_rows(s, case, i, case["path"]).unflatten(1, (-1, group)) - lse[..., None]).sum(2)
        path = s["path_rows"][i] if case["path"] else list(range(case["n"]))
        got[i, :, :ctx] = case["decay"] * got[i, :, :ctx] + p[:, path, :ctx].sum(1)
        if case["path"]:
            for t, node in enumerate(path):
                got[i, :, ctx + t] = p[:, path, ctx + node].sum(1)
    return {"weights": got}
