"""The paged cache and the attention that reads it, as cases that can be timed.

A case is one pass through one operator on device-resident tensors: `write` stores the rows of new
tokens in the pages of their sequences (with an e4m3 cache: quantised, a power-of-two scale to each
row and head), `read` brings rows back into a dense cache, `attend` lets a chunk of new tokens attend
over the pages, and `window` does so where a token sees a sliding window and the first rows.

Row r of sequence s lies in page table[s][r // page] at slot r % page; a sequence's new tokens are the
last rows of its cache.  An e4m3 row holds codes c and one exponent k: its values are c * 2**k, k being
the smallest with max|x| <= 448 * 2**k (and -117 <= k <= 120), kept as the byte k + 127.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f32": 4, "e4m3": 1}
LEAST, MOST = -117, 120   # exponents of an e4m3 row's scale


def _case(name, kind, seqs, heads, kv_heads, dim, dtype, cache, page, length, new, *, ragged=False, packed=False,
          causal=False, window=0, sinks=0, keep=0):
    """length: cached rows of the longest sequence, its new tokens among them; new: new tokens of a sequence, the most of
    any where they are ragged; keep: rows of a list that `read` is given (0: all rows)."""
    return {"name": name, "kind": kind, "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "cache": cache, "page": page, "length": length, "new": new, "ragged": ragged, "packed": packed,
            "causal": causal, "window": window, "sinks": sinks, "keep": keep}


def listed():
    return [
        # one token of each of 32 sequences joins the cache: the call itself is the cost
        _case("write_tokens_e4m3", "write", 32, 32, 8, 128, "bf16", "e4m3", 16, 1200, 1, ragged=True, packed=True),
        # a 48 x 48 map of sixteen sequences (guidance rows among them) joins a layer's cache in 8 bits
        _case("write_map_e4m3", "write", 16, 16, 16, 128, "bf16", "e4m3", 64, 2632, 2304),
        # that layer's whole cache comes back for the step that ranks it
        _case("read_layer_e4m3", "read", 16, 16, 16, 128, "bf16", "e4m3", 64, 3350, 0),
        # the rows that a ranking has kept, out of a cache that is not quantised; odd numbers of rows
        _case("read_kept_bf16", "read", 3, 20, 20, 64, "bf16", "bf16", 32, 1733, 0, keep=433),
        # the last map of an image, 64 x 64 tokens that all see each other and the kept rows, eight sequences
        _case("attend_map", "attend", 8, 16, 16, 128, "bf16", "bf16", 64, 4420, 4096),
        # chunks of prompts of different lengths, four query heads to a KV head, in 8 bits
        _case("attend_chunk_causal_e4m3", "attend", 4, 32, 8, 128, "bf16", "e4m3", 16, 8192, 512, ragged=True,
              packed=True, causal=True),
        # single tokens of many sequences of different lengths, in 8 bits: serving
        _case("attend_tokens_e4m3", "attend", 64, 32, 8, 128, "bf16", "e4m3", 16, 4000, 1, ragged=True, packed=True,
              causal=True),
        # single tokens over two very long caches: the key axis has to be split
        _case("attend_token_long", "attend", 2, 32, 8, 128, "bf16", "bf16", 128, 131072, 1, causal=True),
        # full precision, as when results are checked against the bf16 run; narrow heads
        _case("attend_chunk_f32", "attend", 2, 12, 12, 64, "f32", "f32", 16, 585, 145, causal=True),
        # a chunk of a long prompt where a token sees 1024 rows and four sinks
        _case("window_chunk", "window", 2, 32, 8, 128, "bf16", "bf16", 64, 16384, 2048, causal=True, window=1024,
              sinks=4),
        # single tokens that see a window and sinks, narrow heads, in 8 bits
        _case("window_tokens_e4m3", "window", 48, 16, 16, 64, "bf16", "e4m3", 32, 20000, 1, ragged=True, packed=True,
              causal=True, window=2048, sinks=16),
        # one sequence, one token, a short cache: the smallest call
        _case("window_token_batch1", "window", 1, 16, 16, 128, "bf16", "bf16", 64, 700, 1, causal=True, window=256,
              sinks=4),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = [work(c) for c in listed()]
    most = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        kind = rng.choice(("write", "read", "attend", "attend", "attend", "window", "window"))
        dtype = rng.choice(("bf16", "bf16", "bf16", "bf16", "f32"))
        kv_heads = rng.choice((1, 2, 4, 8, 12, 16, 20, 32))
        case = _case("", kind, _log_int(rng, 1, 64), kv_heads * rng.choice((1, 1, 2, 4, 8)), kv_heads,
                     rng.choice((64, 128, 128)), dtype, rng.choice((dtype, "e4m3")), rng.choice((16, 32, 64, 128, 256)),
                     _log_int(rng, 1, 131072), 0, ragged=rng.random() < 0.5)
        del case["name"]
        if kind == "read":
            case["heads"] = kv_heads * rng.choice((1, 1, 1, 2, 4)) if kv_heads < 16 else kv_heads
            case["keep"] = rng.choice((0, 0, max(1, case["length"] // rng.randint(3, 20))))
            if case["keep"]:
                case["ragged"] = False
        else:
            case["new"] = rng.choice((1, 1, _log_int(rng, 1, 4096)))
            case["length"] = max(case["length"], case["new"])
            case["packed"] = rng.random() < 0.5
        if kind == "attend":
            case["causal"] = rng.random() < 0.6
        if kind == "window":
            case.update(causal=rng.random() < 0.8, window=_log_int(rng, 1, 8192), sinks=rng.choice((0, 1, 4, 64, 300)))
        w = work(case)
        scores = case["seqs"] * case["heads"] * case["new"] * case["length"]
        cached = case["seqs"] * case["kv_heads"] * case["length"] * case["dim"]
        if w["bytes"] <= most["bytes"] and cached <= 1 << 28 and scores <= 3 << 29 and \
                w["flops"] <= most["flops"] / (20 if dtype == "f32" else 1):
            return case


# ---- a case's lengths: the same for every seed, so that its work is known

def _lengths(case):
    """(cached rows, new tokens) of each sequence."""
    r = random.Random("%(seqs)d %(length)d %(new)d %(page)d" % case)
    got = []
    for s in range(case["seqs"]):
        length, new = case["length"], case["new"]
        if case["ragged"] and s:
            new = r.randint(1, new) if new else 0
            length = r.randint(min(length, max(new, length // 16)), length)
        got.append((length, new))
    return got


def _seen(case, p, length):
    """Rows [0, a) and [b, c) that a token at position p sees."""
    c = min(p + 1, length) if case["causal"] else length
    b = max(0, p - case["window"] + 1) if case["kind"] == "window" else 0
    a = min(case["sinks"], b, c) if case["kind"] == "window" else 0
    return a, b, c


def work(case):
    e, d, ec = BYTES[case["dtype"]], case["dim"], BYTES[case["cache"]]
    row = case["kv_heads"] * (d * ec + (1 if case["cache"] == "e4m3" else 0))   # one cached row of K or of V
    lens = _lengths(case)
    new = sum(n for _, n in lens)
    if case["kind"] == "write":
        return {"bytes": 2 * new * (case["kv_heads"] * d * e + row), "flops": 0}
    if case["kind"] == "read":
        out = case["keep"] * case["seqs"] if case["keep"] else sum(length for length, _ in lens)
        listing = 4 * out * case["heads"] if case["keep"] else 0
        # where rows are listed each head may ask for others
        return {"bytes": 2 * out * (row * (case["heads"] // case["kv_heads"] if case["keep"] else 1)
                                    + case["heads"] * d * e) + listing, "flops": 0}
    rows = pairs = 0
    for length, n in lens:
        first, last = _seen(case, length - n, length), _seen(case, length - 1, length)
        rows += min(last[2], max(first[0], last[0]) + last[2] - first[1]) if case["kind"] == "window" else length
        if case["kind"] == "attend":
            pairs += n * length - (n * (n - 1) // 2 if case["causal"] else 0)
        else:
            for t in range(n):
                a, b, c = _seen(case, length - n + t, length)
                pairs += a + max(0, c - b)
    return {"bytes": 2 * rows * row + 2 * new * case["heads"] * d * e, "flops": 4 * d * pairs * case["heads"]}


# ---- inputs

class _Values:
    """Queries, keys and values that share a rank-8 subspace per KV head, as trained ones do: peaked attention."""

    def __init__(self, case, seed):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.dim = case["dim"]
        self.w = self.normal(case["kv_heads"], 8, self.dim) / math.sqrt(8.0)

    def normal(self, *size):
        return torch.randn(*size, device="cuda", dtype=torch.float32, generator=self.gen)

    def rows(self, n, per):
        """[n, KV heads, per, d]"""
        h = self.w.shape[0]
        return self.normal(n, h, per, self.dim) + torch.matmul(self.normal(n, h, per, 8), self.w)


def _power(k):
    """2**k as fp32, from the bits."""
    return ((k + 127) << 23).view(torch.float32)


def _quantised(x):
    """codes and exponent bytes of rows in the last dimension, elementary operations in fp32 (all exact but the rounding)."""
    x = x.float()
    finite = torch.isfinite(x)
    mant, exp = torch.frexp(torch.where(finite, x.abs(), 0.0).amax(-1, keepdim=True))
    k = torch.where(mant <= 0.875, exp - 9, exp - 8).clamp(LEAST, MOST)
    k = torch.where(mant == 0, LEAST, k).int()
    most = torch.where(k == MOST, 240.0, 448.0)     # above 240 * 2**120 a value would round to 2**128
    y = torch.minimum(torch.maximum(x * _power(-k), -most), most)
    y = torch.where(finite, y, float("nan"))
    return y.to(torch.float8_e4m3fn), (k + 127).to(torch.uint8).squeeze(-1)


def _pool(case, values, n_page):
    """Pages of K or V, and their scales."""
    x = values.rows(n_page, case["page"])
    if case["cache"] != "e4m3":
        return x.to(DTYPES[case["cache"]]), None
    return _quantised(x.to(DTYPES[case["dtype"]]))


def prepare(case, seed):
    values, lens = _Values(case, seed), _lengths(case)
    page, seqs, dtype = case["page"], case["seqs"], DTYPES[case["dtype"]]
    width = -(-case["length"] // page)
    used = [-(-length // page) for length, _ in lens]
    n_page = sum(used) + max(1, sum(used) // 16)    # some pages belong to nobody
    order = torch.randperm(n_page, device="cuda", generator=values.gen, dtype=torch.int32)
    table = torch.full((seqs, width), -1, device="cuda", dtype=torch.int32)
    at = 0
    for s in range(seqs):
        table[s, :used[s]] = order[at:at + used[s]]
        at += used[s]
    state = {"case": case, "table": table, "lens": torch.tensor([n for n, _ in lens], device="cuda", dtype=torch.int32),
             "count": torch.tensor([n for _, n in lens], device="cuda", dtype=torch.int32),
             "first": None, "new": case["new"], "scale": case["dim"] ** -0.5}
    state["k"], state["k_scale"] = _pool(case, values, n_page)
    state["v"], state["v_scale"] = _pool(case, values, n_page)
    if case["kind"] == "read":
        rows = case["keep"] or case["length"]
        size = seqs, case["heads"], rows, case["dim"]
        state["k_dst"], state["v_dst"] = (torch.zeros(size, device="cuda", dtype=dtype) for _ in range(2))
        state["idx"] = None
        if case["keep"]:
            pick = torch.rand(seqs, case["heads"], case["length"], device="cuda", generator=values.gen)
            state["idx"] = pick.topk(rows, -1).indices.sort(-1).values.int()
    else:
        if case["packed"]:   # the tokens of all sequences one behind the other
            counts = [n for _, n in lens]
            state["first"] = torch.tensor([sum(counts[:s]) for s in range(seqs)], device="cuda", dtype=torch.int32)
            shapes = {h: (sum(counts), h, case["dim"]) for h in (case["heads"], case["kv_heads"])}
        else:
            shapes = {h: (seqs, h, case["new"], case["dim"]) for h in (case["heads"], case["kv_heads"])}

        def rows_of(h):
            g = h // case["kv_heads"]
            if case["packed"]:
                x = values.rows(shapes[h][0], g)                                  # [tokens, KV heads, group, d]
                return x.reshape(shapes[h]).to(dtype)
            x = values.rows(seqs, g * case["new"])                                # [S, KV heads, group * n, d]
            return x.reshape(shapes[h]).to(dtype)

        if case["kind"] == "write":
            state["k_new"], state["v_new"] = rows_of(case["kv_heads"]), rows_of(case["kv_heads"])
        else:
            state["q"] = rows_of(case["heads"])
            state["out"] = torch.zeros_like(state["q"])
    if own:
        import paper_2505_19602_amd as skv
        state["shape"] = skv.Shape(seqs, case["heads"], case["dim"], dtype)
        state["pages"] = skv.Pages(state["k"], state["v"], table, state["lens"], state["k_scale"], state["v_scale"])
        if case["kind"] in ("attend", "window"):
            need = skv.pages_workspace_bytes(state["shape"], state["pages"], case["new"], causal=case["causal"],
                                             window=case["window"], n_sink=case["sinks"])
            state["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    return state


# ---- the framework's calls

def _own_run(s):
    import paper_2505_19602_amd as skv
    case = s["case"]
    chunk = {"first": s["first"], "count": s["count"], "max_new": s["new"]}
    if case["kind"] == "write":
        skv.pages_write(s["shape"], s["pages"], s["k_new"], s["v_new"], **chunk)
        return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if case["kind"] == "read":
        skv.pages_read(s["shape"], s["pages"], s["idx"], s["k_dst"].shape[2], s["k_dst"], s["v_dst"])
        return {"k": s["k_dst"], "v": s["v_dst"]}
    skv.pages_attend(s["shape"], s["pages"], s["q"], s["out"], s["ws"], causal=case["causal"], window=case["window"],
                     n_sink=case["sinks"], **chunk)
    return {"out": s["out"]}


# ---- the plain forms

def _places(s, positions):
    """Page and slot of positions [S, ...]."""
    page = s["case"]["page"]
    flat = positions.reshape(positions.shape[0], -1)
    pid = s["table"].gather(1, (flat // page).clamp(0, s["table"].shape[1] - 1)).reshape(positions.shape)
    return pid.long().clamp(min=0), (positions % page).long()


def _gathered(s, name, pid, slot, heads=None):
    """fp32 values of cached rows: pid, slot [S, L] -> [S, L, KV heads, d]; with heads [S, H, L] of one head each."""
    pool = s[name]
    at = (pid, slice(None), slot) if heads is None else (pid, heads, slot)
    if s["case"]["cache"] != "e4m3":
        return pool[at].float()
    codes = pool.view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
    return codes * _power(s[name + "_scale"][at].int() - 127).unsqueeze(-1)


def _token_rows(s, x):
    """Rows of the chunk as [S, heads, n, d], whatever lies behind a sequence's tokens."""
    if s["first"] is None:
        return x
    at = s["first"].long()[:, None] + torch.arange(s["new"], device=x.device)
    return x[at.clamp(max=x.shape[0] - 1)].transpose(1, 2)


def _plain_write(s):
    case = s["case"]
    t = torch.arange(s["new"], device="cuda", dtype=torch.int32)[None]
    live = t < s["count"][:, None]
    pid, slot = _places(s, (s["lens"] - s["count"])[:, None] + t)
    pid, slot = pid[live], slot[live]
    for name in ("k", "v"):
        x = _token_rows(s, s[name + "_new"]).transpose(1, 2)[live]      # [tokens, KV heads, d]
        if case["cache"] == "e4m3":
            codes, scale = _quantised(x)
            s[name].view(torch.uint8)[pid, :, slot] = codes.view(torch.uint8)
            s[name + "_scale"][pid, :, slot] = scale
        else:
            s[name][pid, :, slot] = x
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _plain_read(s):
    case = s["case"]
    group = case["heads"] // case["kv_heads"]
    if s["idx"] is None:
        pos = torch.arange(case["length"], device="cuda", dtype=torch.int32)[None].expand(case["seqs"], -1)
        pid, slot = _places(s, pos)
        live = (pos < s["lens"][:, None])[:, None, :, None]
    else:
        pid, slot = _places(s, s["idx"])
        heads = (torch.arange(case["heads"], device="cuda") // group)[None, :, None]
    for name in ("k", "v"):
        dst = s[name + "_dst"]
        if s["idx"] is None:
            x = _gathered(s, name, pid, slot).transpose(1, 2).repeat_interleave(group, 1)
            dst.copy_(torch.where(live, x.to(dst.dtype), dst))
        else:
            dst.copy_(_gathered(s, name, pid, slot, heads).to(dst.dtype))
    return {"k": s["k_dst"], "v": s["v_dst"]}


def _plain_attend(s):
    case = s["case"]
    seqs, heads, kv_heads, n, d = case["seqs"], case["heads"], case["kv_heads"], s["new"], case["dim"]
    j = torch.arange(case["length"], device="cuda", dtype=torch.int32)
    pid, slot = _places(s, j[None].expand(seqs, -1))
    k = _gathered(s, "k", pid, slot).permute(0, 2, 3, 1).contiguous()    # [S, KV heads, d, L]
    v = _gathered(s, "v", pid, slot).transpose(1, 2).contiguous()        # [S, KV heads, L, d]
    q = _token_rows(s, s["q"]).float().reshape(seqs, kv_heads, heads // kv_heads * n, d)
    w = torch.matmul(q * s["scale"], k).reshape(seqs, heads, n, -1)
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    p = ((s["lens"] - s["count"])[:, None] + t)[:, :, None]              # [S, n, 1]
    sees = (j < s["lens"][:, None, None]).expand(seqs, n, -1)
    if case["causal"]:
        sees = sees & (j <= p)
    if case["kind"] == "window":
        sees = sees & ((j > p - case["window"]) | (j < case["sinks"]))
    w.masked_fill_(~sees[:, None], float("-inf"))
    w.sub_(w.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w.reshape(seqs, kv_heads, -1, w.shape[-1]), v).reshape(seqs, heads, n, d)
    out = torch.where(total > 0, out / total, 0.0).to(s["out"].dtype)
    live = t < s["count"][:, None]
    if s["first"] is None:
        s["out"].copy_(torch.where(live[:, None, :, None], out, s["out"]))
    else:
        s["out"][(s["first"][:, None] + t)[live].long()] = out.transpose(1, 2)[live]
    return {"out": s["out"]}


def run(state):
    if own:
        return _own_run(state)
    kind = state["case"]["kind"]
    return (_plain_write if kind == "write" else _plain_read if kind == "read" else _plain_attend)(state)


# ---- the definitions in 64 bits

def _exact_power(k):
    """2**k in 64 bits: the functions of the GPU are an ulp off here, and a tie of a rounding is not one any more."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x):
    """e4m3 codes of rows, in 64 bits."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    k = torch.ceil(torch.log2(top.clamp(min=2.0 ** -200) / 448.0)).clamp(LEAST, MOST)
    k = torch.where(top > 448.0 * _exact_power(k), k + 1, k)             # (the logarithm's own rounding)
    k = torch.where((top <= 448.0 * _exact_power(k - 1)) & (k > LEAST), k - 1, k)
    y = x / _exact_power(k)
    _, exp = torch.frexp(y.abs().clamp(min=2.0 ** -6))
    step = _exact_power(exp - 4)
    return torch.round(y / step) * step


def _exact_rows(s, name, seq):
    """All cached rows of a sequence, [KV heads, rows, d] in 64 bits."""
    n = int(s["lens"][seq])
    pages = s["table"][seq, :-(-n // s["case"]["page"])].long()
    x = s[name][pages].double()                                          # [pages, KV heads, page, d]
    if s["case"]["cache"] == "e4m3":
        x = x * _exact_power(s[name + "_scale"][pages].int() - 127)[..., None]
    return x.transpose(0, 1).flatten(1, 2)[:, :n]


def _tokens_of(s, seq):
    """Where the new tokens of a sequence lie: an index into q, k_new, v_new or out, and their number."""
    n = int(s["count"][seq])
    if s["first"] is None:
        return (seq, slice(None), slice(0, n)), n
    at = int(s["first"][seq])
    return slice(at, at + n), n


def exact(case, seed):
    s = prepare(case, seed)
    seqs, group = case["seqs"], case["heads"] // case["kv_heads"]
    if case["kind"] == "write":
        got = {"k": s["k"].double(), "v": s["v"].double(), "k_scale": None, "v_scale": None}
        for seq in range(seqs):
            at, n = _tokens_of(s, seq)
            for i in range(n):
                r = int(s["lens"][seq]) - n + i
                if i == 0 or r % case["page"] == 0:                      # the tokens that share a page
                    m = min(n - i, case["page"] - r % case["page"])
                    pid, slot = int(s["table"][seq, r // case["page"]]), r % case["page"]
                    for name in ("k", "v"):
                        x = s[name + "_new"][at]
                        x = x if s["first"] is None else x.transpose(0, 1)   # [KV heads, tokens, d]
                        x = x[:, i:i + m].double()
                        got[name][pid, :, slot:slot + m] = _exact_codes(x) if case["cache"] == "e4m3" else x
        return got
    if case["kind"] == "read":
        got = {"k": s["k_dst"].double(), "v": s["v_dst"].double()}
        for seq in range(seqs):
            for name in ("k", "v"):
                x = _exact_rows(s, name, seq).repeat_interleave(group, 0)
                if s["idx"] is not None:
                    x = x.gather(1, s["idx"][seq].long()[..., None].expand(-1, -1, case["dim"]))
                got[name][seq, :, :x.shape[1]] = x
        return got
    out = s["out"].double()
    for seq in range(seqs):
        at, n = _tokens_of(s, seq)
        k, v = _exact_rows(s, "k", seq), _exact_rows(s, "v", seq)
        q = s["q"][at].double()
        q = q if s["first"] is None else q.transpose(0, 1)               # [heads, tokens, d]
        length = k.shape[1]
        j, p = torch.arange(length, device="cuda"), torch.arange(length - n, length, device="cuda")[:, None]
        hidden = (j > p) if case["causal"] else torch.zeros(n, length, dtype=torch.bool, device="cuda")
        if case["kind"] == "window":
            hidden = hidden | ((j <= p - case["window"]) & (j >= case["sinks"]))
        for h in range(case["heads"]):
            w = torch.matmul(q[h], k[h // group].t()) / math.sqrt(case["dim"])
            w = torch.softmax(w.masked_fill(hidden, float("-inf")), -1)
            o = torch.matmul(torch.nan_to_num(w, nan=0.0), v[h // group])
            if s["first"] is None:
                out[seq, h, :n] = o
            else:
                out[at, h] = o
    return {"out": out}
