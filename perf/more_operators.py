"""The operators that keep a cache within a budget, as this library's speed is measured on them.

One case is one call of one operator for one attention layer:

* ``window``   attention with a sliding window and attention sinks over the paged
  cache (``kf.window_attn``): a row at position p sees the tokens t <= p with
  t < sinks or t > p - window; sequence b has ``rows`` rows behind ``ctx`` cached
  tokens (one row: a decode step; many: a prompt, whole or in chunks);
* ``weights``  the attention weight that each cached token and KV head receives from
  the rows' softmax, added to what it received before (``kf.attn_weights``):
  ``decay`` times the old value plus the sum over rows and the group's query heads;
  a token that is new in the call (its own row is among the rows) starts from 0;
* ``evict``    eviction from the cache by accumulated weight (``kf.kv_evict``): of
  each sequence's ``ctx`` tokens at most ``keep`` stay per KV head, the first
  ``first``, the last ``last`` and the heaviest of the others, moved in their order
  into the pages of a route of their own.

Lengths are log-uniform in ``lo .. hi`` (``lens`` seeds them, so that a case
always has the same ones), cut into routes of ``part`` tokens.  Pools hold bf16,
or E4M3 codes with one scale per page and KV head (``fp8``); ``head_major``
pools or page-major, ``permuted`` page ids (a pool after some churn) or
contiguous ones.

The plain forms work on sequences padded to the longest, without a loop over
them.
"""
from __future__ import annotations

import math
import random

import torch

own = False

PAGE, DIM = 16, 128
SCALE = 1.0 / math.sqrt(DIM)
DEVICE = "cuda"


def _case(name, op, seqs, q_heads, kv_heads, rows, ctx, part, *, sinks=0, window=0, decay=0.0,
          keep=0, first=0, last=0, fp8=False, head_major=False, permuted=False, lens=1):
    return {"name": name, "op": op, "seqs": seqs, "q_heads": q_heads, "kv_heads": kv_heads,
            "rows_lo": rows[0], "rows_hi": rows[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "part": part, "sinks": sinks, "window": window, "decay": decay, "keep": keep,
            "first": first, "last": last, "fp8": fp8, "head_major": head_major,
            "permuted": permuted, "lens": lens}


def listed():
    return [
        # the smallest decode step: one chat on a small layer, latency only
        _case("window_tiny", "window", 1, 8, 2, (1, 1), (700, 700), 2048, sinks=4, window=256),
        # decode steps of agentic requests of 2K .. 64K tokens in one permuted pool
        _case("window_decode", "window", 48, 32, 8, (1, 1), (2048, 65536), 16384, sinks=4,
              window=4096, permuted=True),
        # one long document, 16K tokens, on a Llama-3.1-8B layer
        _case("window_prompt", "window", 1, 32, 8, (16384, 16384), (0, 0), 8192, sinks=4,
              window=2048),
        # chunked prefill: ~500 rows of each request behind ~30K cached tokens, fp8, 64/8 heads
        _case("window_chunk_fp8", "window", 4, 64, 8, (400, 512), (20000, 32768), 16384, sinks=64,
              window=8000, fp8=True, permuted=True),
        # the weights of a small layer's decode step
        _case("weights_tiny", "weights", 1, 8, 2, (1, 1), (700, 700), 2048, decay=1.0),
        # the decode step of a Llama-3.1-8B layer at 32K tokens
        _case("weights_decode", "weights", 16, 32, 8, (1, 1), (32767, 32767), 8192, decay=1.0),
        # the last 32 rows of prompts of 2K .. 32K tokens look at the whole prompt, fp8 pages
        _case("weights_observe_fp8", "weights", 8, 64, 8, (32, 32), (2000, 32000), 16384, fp8=True,
              permuted=True),
        # every row of one prompt of 10K tokens
        _case("weights_prompt", "weights", 1, 32, 8, (9973, 9973), (0, 0), 8192),
        # the smallest eviction: one chat back to 256 tokens
        _case("evict_tiny", "evict", 1, 8, 2, (0, 0), (700, 700), 2048, keep=256, first=4, last=64),
        # agentic requests of 2K .. 64K tokens down to 4096 each, half of them the latest
        _case("evict_agentic", "evict", 48, 32, 8, (0, 0), (2048, 65536), 16384, keep=4096,
              first=4, last=2048, permuted=True),
        # a 70B-like layer (64/8 heads) with fp8 K/V, 16K tokens down to 3000
        _case("evict_fp8", "evict", 16, 64, 8, (0, 0), (16000, 16000), 8192, keep=3000, first=16,
              last=256, fp8=True),
        # one document of 128K tokens down to 16K
        _case("evict_long", "evict", 1, 32, 8, (0, 0), (131072, 131072), 16384, keep=16384,
              first=4, last=1024),
    ]


_HEADS = ((8, 2), (16, 2), (32, 8), (64, 8), (32, 32), (40, 8), (24, 8), (64, 4), (8, 1), (16, 16))


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {op: max(_cost(work(c)) for c in listed() if c["op"] == op)
            for op in ("window", "weights", "evict")}
    while True:
        op = rng.choice(("window", "weights", "evict"))
        q_heads, kv_heads = rng.choice(_HEADS)
        lo = 1 if rng.random() < 0.4 else spread(1, 8000)
        hi = lo if rng.random() < 0.4 else min(16384, spread(lo, 20 * lo))
        clo = spread(1, 60000) if lo < 600 or rng.random() < 0.3 else 0
        chi = clo if rng.random() < 0.3 else min(65536, spread(max(1, clo), 20 * max(1, clo)))
        more = {}
        if op == "window":
            more = {"sinks": rng.choice((0, 1, 4, 16, 64, 300)), "window": spread(1, 16000)}
        elif op == "weights":
            more = {"decay": rng.choice((0.0, 0.5, 1.0))}
        else:
            lo = hi = 0
            clo, chi = max(1, clo), max(1, chi)
            keep = spread(1, 16384)
            more = {"keep": keep, "first": rng.choice((0, 1, 4, 16)),
                    "last": rng.choice((0, keep // 16, keep // 2, keep))}
        c = _case("", op, spread(1, 64), q_heads, kv_heads, (min(lo, hi), hi),
                  (min(clo, chi), chi), rng.choice((2048, 4096, 8192, 16384)),
                  fp8=rng.random() < 0.35, head_major=rng.random() < 0.25,
                  permuted=rng.random() < 0.6, lens=rng.randrange(1 << 20), **more)
        del c["name"]
        # the padded plain forms hold every sequence at the longest one's length
        n, t = _longest(c)
        if c["seqs"] * t * kv_heads > 1 << 25 or c["seqs"] * q_heads * n * t > 9e9:
            continue
        if 2e4 <= _cost(work(c)) <= most[op]:
            return c


def _cost(w):
    return max(w["bytes"], w["flops"] / 150)


# ------------------------------------------------------------------- tables
def _lengths(case):
    """(cached tokens, rows) of each sequence."""
    rng = random.Random(case["lens"])

    def one(lo, hi):
        if lo < 1:
            return rng.randint(lo, hi)
        return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    return [(one(case["ctx_lo"], case["ctx_hi"]), one(case["rows_lo"], case["rows_hi"]))
            for _ in range(case["seqs"])]


def _longest(case):
    """The most rows of a sequence, and the most tokens that it holds."""
    lens = _lengths(case)
    return max(n for _, n in lens), max(c + n for c, n in lens)


def _table(case):
    """Route rows [seq, part, tok_begin, tok_end, page_base, page_cap] and the CSR rows
    of the sequences.  An eviction's sequences end in an empty route for what is kept."""
    rows, begin, base = [], [0], 0
    for b, (c, n) in enumerate(_lengths(case)):
        for k, t0 in enumerate(range(0, max(c + n, 1), case["part"])):
            t1 = min(t0 + case["part"], c + n)
            cap = -(-(t1 - t0) // PAGE)
            rows.append([b, k, t0, t1, base, cap])
            base += cap
        if case["op"] == "evict":
            cap = -(-min(c, case["keep"]) // PAGE)
            rows.append([b, len(rows) - begin[-1], 0, 0, base, cap])
            base += cap
        begin.append(len(rows))
    return rows, begin


def _csr(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _page_ids(case, caps, gen):
    """Page ids of the routes, route after route, and the pool's page count."""
    total = sum(caps)
    if case["permuted"]:
        return torch.randperm(total, generator=gen, device=DEVICE).to(torch.int32), total
    return torch.arange(total, dtype=torch.int32, device=DEVICE), total


# ------------------------------------------------------------------- inputs
def _pages(case, pool):
    """The pool indexed by page first, whatever its layout."""
    return pool.transpose(0, 1) if case["head_major"] else pool


def _code(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _decode(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _pool(case, P, inner, gen):
    """A pool of N(0, 1) values in its storage layout, and its scales (fp8):
    pages as appends leave them, their first token's largest value at 28."""
    H = case["kv_heads"]
    lead = (H, P) if case["head_major"] else (P, H)
    if not case["fp8"]:
        return torch.randn(lead + inner, generator=gen, device=DEVICE, dtype=torch.bfloat16), None
    pool = torch.empty(lead + inner, device=DEVICE, dtype=torch.uint8)
    scale = torch.empty((P, H), device=DEVICE)
    step = max(1, (1 << 27) // (H * PAGE * DIM))
    for p in range(0, P, step):
        x = torch.randn((min(step, P - p), H) + inner, generator=gen, device=DEVICE)
        first = x[:, :, 0] if inner[0] == PAGE else x[:, :, :, 0]
        s = first.abs().amax(2) / 28.0
        scale[p:p + len(s)] = s
        _pages(case, pool)[p:p + len(s)] = _code(x / s[:, :, None, None])
    return pool, scale


def _inputs(case, seed):
    """The call's inputs on the GPU, from the seed alone."""
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    rows, begin = _table(case)
    lens = _lengths(case)
    B, Hq, H = case["seqs"], case["q_heads"], case["kv_heads"]
    N = sum(n for _, n in lens)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEVICE)

    x = {"routes": ints(rows), "seq_route_begin": ints(begin)}
    x["page_ids"], P = _page_ids(case, [r[5] for r in rows], gen)
    x["k_pool"], x["k_scale"] = _pool(case, P, (PAGE, DIM), gen)
    if case["op"] != "weights":
        x["v_pool"], x["v_scale"] = _pool(case, P, (DIM, PAGE), gen)
    if case["op"] != "window":
        # a few tokens took most of the weight, many hardly any, some none
        u = torch.rand((P, H, PAGE), generator=gen, device=DEVICE)
        x["weights"] = torch.where(u < 0.05, 0.0, u ** 12 * 8.0)
    if case["op"] == "evict":
        x["into"] = ints([e - 1 for e in begin[1:]])
        x["keep"] = ints([case["keep"]] * B)
        return x
    x["q"] = torch.randn((N, Hq, DIM), generator=gen, device=DEVICE, dtype=torch.bfloat16)
    row_begin = _csr([n for _, n in lens])
    x["seq_row_begin"] = ints(row_begin)
    x["first_pos"] = ints([c for c, _ in lens])
    # an attention sink: the first token of each sequence scores about 7 for the first
    # row's heads
    first = x["page_ids"][torch.tensor([rows[r][4] for r in begin[:-1]], device=DEVICE)].long()
    q = x["q"][torch.tensor(row_begin[:-1], device=DEVICE)]
    sink = 0.6 * q.view(B, H, Hq // H, DIM).float().sum(2)
    pages = _pages(case, x["k_pool"])
    if case["fp8"]:
        pages[first, :, 0] = _code(sink / x["k_scale"][first][:, :, None])
    else:
        pages[first, :, 0] = sink.to(torch.bfloat16)
    if case["op"] == "weights":
        x["lse"] = _row_lse(case, x, rows, begin, lens)
    return x


def _row_lse(case, x, rows, begin, lens):
    """What the layer's attention left of its softmax: ln sum exp(s) of each row and head."""
    H, G = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    lse = torch.empty((x["q"].shape[0], H, G), device=DEVICE)
    at = 0
    for b, (c, n) in enumerate(lens):
        ids = torch.cat([x["page_ids"][r[4]:r[4] + r[5]] for r in rows[begin[b]:begin[b + 1]]]).long()
        k = _pages(case, x["k_pool"])[ids]                       # [pages, H, 16, 128]
        k = _decode(k) * x["k_scale"][ids][..., None, None] if case["fp8"] else k.float()
        k = k.transpose(0, 1).reshape(H, -1, DIM)
        # (pages at the end of a route that is no multiple of 16 would leave a gap)
        t = torch.cat([torch.arange(r[2], r[2] + PAGE * r[5], device=DEVICE)
                       for r in rows[begin[b]:begin[b + 1]]])
        k = k.transpose(1, 2).contiguous()
        for i0 in range(0, n, 1024):
            i1 = min(n, i0 + 1024)
            q = x["q"][at + i0:at + i1].float().view(i1 - i0, H, G, DIM).transpose(0, 1)
            s = torch.matmul(q.reshape(H, -1, DIM), k).mul_(SCALE).view(H, i1 - i0, G, -1)
            p = c + torch.arange(i0, i1, device=DEVICE)
            s.masked_fill_((t > p[:, None])[:, None, :], -math.inf)
            lse[at + i0:at + i1] = torch.logsumexp(s, -1).transpose(0, 1)
        at += n
    return lse.view(-1, H * G)


def prepare(case, seed):
    x = _inputs(case, seed)
    st = {"case": dict(case), "x": x, "err": torch.zeros(1, dtype=torch.int32, device=DEVICE),
          "most_pages": max(r[5] for r in _table(case)[0]), "longest": _longest(case)}
    if case["op"] == "window":
        N, Hq = x["q"].shape[:2]
        st["out"] = torch.empty((N, Hq, DIM), device=DEVICE, dtype=torch.bfloat16)
        st["lse"] = torch.empty((N, Hq), device=DEVICE)
    elif case["op"] == "weights":
        st["weights"] = x["weights"].clone()
    else:
        st["routes"] = x["routes"].clone()
    return st


# ---------------------------------------------------------------------- run
def run(st):
    case, x = st["case"], st["x"]
    if case["op"] == "window":
        if own:
            _call(st)()
        else:
            _window_plain(st)
        return {"out": st["out"], "lse": st["lse"]}
    if case["op"] == "weights":
        if case["decay"] != 0.0:
            st["weights"].copy_(x["weights"])   # what earlier steps left
        if own:
            _call(st)()
        else:
            _weights_plain(st)
        return {"weights": st["weights"]}
    st["routes"].copy_(x["routes"])             # the step's route table
    if own:
        _call(st)()
    else:
        _evict_plain(st)
    got = {"routes": st["routes"], "k_pool": x["k_pool"], "v_pool": x["v_pool"],
           "weights": x["weights"]}
    if case["fp8"]:
        got.update(k_pool=x["k_pool"].view(torch.float8_e4m3fn),
                   v_pool=x["v_pool"].view(torch.float8_e4m3fn),
                   k_scale=x["k_scale"], v_scale=x["v_scale"])
    return got


def _call(st):
    """The operator bound to the state's buffers, as a serving loop keeps it: its
    arguments are checked and marshalled once."""
    if "call" not in st:
        from paper_2606_29207_amd import kf
        case, x = st["case"], st["x"]
        H, P = case["kv_heads"], x["k_pool"].shape[1 if case["head_major"] else 0]
        shape = kf.make_shape(case["seqs"], case["q_heads"], H,
                              kf.KV_FP8_E4M3 if case["fp8"] else kf.KV_BF16, P,
                              x["page_ids"].numel(), SCALE,
                              kf.KV_HEAD_MAJOR if case["head_major"] else kf.KV_PAGE_MAJOR)
        if case["op"] == "window":
            ws = kf.alloc_rows_workspace(shape, x["q"].shape[0], DEVICE)
            st["call"] = kf.bind_window_attn(
                shape, x["q"], x["first_pos"], case["sinks"], case["window"], x["k_pool"],
                x["v_pool"], x["routes"], st["most_pages"], x["page_ids"], x["seq_route_begin"],
                x["seq_row_begin"], st["out"], st["lse"], ws, st["err"], k_scale=x["k_scale"],
                v_scale=x["v_scale"])
        elif case["op"] == "weights":
            st["call"] = kf.bind_attn_weights(
                shape, x["q"], x["lse"], x["first_pos"], x["k_pool"], x["routes"],
                st["most_pages"], x["page_ids"], x["seq_row_begin"], case["decay"], st["weights"],
                st["err"], k_scale=x["k_scale"])
        else:
            st["call"] = kf.bind_kv_evict(
                shape, x["k_pool"], x["v_pool"], x["weights"], st["routes"], st["most_pages"],
                x["page_ids"], x["seq_route_begin"], x["into"], x["keep"], case["keep"],
                case["first"], case["last"], st["err"], k_scale=x["k_scale"],
                v_scale=x["v_scale"])
    return st["call"]


def _places(st):
    """Page ids, slots [B, T] of every sequence's first T tokens, T the longest's (page 0
    behind a sequence's last), and the tokens each one holds."""
    case, x = st["case"], st["x"]
    T = max(1, st["longest"][1])
    begin, held = x["seq_route_begin"].long(), x["held"]
    t = torch.arange(T, device=DEVICE)
    r = torch.minimum(begin[:-1, None] + t // case["part"], begin[1:, None] - 1)
    ok = t < held[:, None]
    j = torch.where(ok, t - x["routes"][r, 2], 0)
    at = x["routes"][r, 4].long() + j // PAGE
    pid = torch.where(ok, x["page_ids"][at.clamp(max=x["page_ids"].numel() - 1)], 0).long()
    return pid, j % PAGE, ok


def _padded(st, pool, scale, is_v, pid, slot):
    """K or V [B, H, T, 128] of those places, 32 bits."""
    pages = _pages(st["case"], pool)
    k = pages[pid, :, :, slot] if is_v else pages[pid, :, slot]   # [B, T, H, 128]
    k = _decode(k) * scale[pid][..., None] if st["case"]["fp8"] else k.float()
    return k.transpose(1, 2).contiguous()


def _rows_padded(st):
    """q [B, H, G n, 128] of every sequence's rows, padded to the most rows n, and the
    places [B, n] of the rows in the packed order."""
    case, x = st["case"], st["x"]
    B, H, n = case["seqs"], case["kv_heads"], st["longest"][0]
    G = case["q_heads"] // H
    begin = x["seq_row_begin"].long()
    row = begin[:-1, None] + torch.arange(n, device=DEVICE)
    real = row < begin[1:, None]
    row = torch.where(real, row, 0)
    q = x["q"][row].float().view(B, n, H, G, DIM).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, DIM)
    return q, row, real


def _held(st):
    x = st["x"]
    if "held" not in x:
        x["held"] = x["routes"][x["seq_route_begin"][1:].long() - 1, 3]
    return x["held"]


def _window_plain(st):
    case, x = st["case"], st["x"]
    B, Hq, H, n = case["seqs"], case["q_heads"], case["kv_heads"], st["longest"][0]
    G = Hq // H
    _held(st)
    q, _, _ = _rows_padded(st)
    pid, slot, ok = _places(st)
    k = _padded(st, x["k_pool"], x["k_scale"], False, pid, slot)
    v = _padded(st, x["v_pool"], x["v_scale"], True, pid, slot)
    t = torch.arange(k.shape[2], device=DEVICE)
    p = (x["first_pos"][:, None] + torch.arange(n, device=DEVICE))[:, :, None]    # [B, n, 1]
    sees = ok[:, None, :] & (t <= p) & ((t < case["sinks"]) | (t > p - case["window"]))
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(SCALE)
    s = s.view(B, H, G, n, -1).masked_fill_(~sees[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=-1e30)
    total = s.sub_(top).exp_().sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, H, G * n, -1), v).view(B, H, G, n, DIM) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, DIM)
    lse = lse.permute(0, 3, 1, 2).reshape(B, n, Hq)
    # the rows of the packed outputs: place e is row e - begin[b] of sequence b
    begin = x["seq_row_begin"].long()
    e = torch.arange(x["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(begin, e, right=True) - 1
    st["out"].copy_(o[b, e - begin[b]])
    st["lse"].copy_(lse[b, e - begin[b]])


def _weights_plain(st):
    case, x = st["case"], st["x"]
    B, Hq, H, n = case["seqs"], case["q_heads"], case["kv_heads"], st["longest"][0]
    G = Hq // H
    x["held"] = x["routes"][x["seq_route_begin"][1:].long() - 1, 3]
    q, row, real = _rows_padded(st)
    pid, slot, ok = _places(st)
    k = _padded(st, x["k_pool"], x["k_scale"], False, pid, slot)
    t = torch.arange(k.shape[2], device=DEVICE)
    p = x["first_pos"][:, None] + torch.arange(n, device=DEVICE)
    sees = (t <= p[:, :, None]) & real[:, :, None]                # [B, n, T]
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(SCALE).view(B, H, G, n, -1)
    lse = x["lse"][row].view(B, n, H, G).permute(0, 2, 3, 1)
    s.sub_(lse[..., None]).masked_fill_(~sees[:, None, None], -math.inf)
    total = s.exp_().sum((2, 3))                                  # [B, H, T]
    pid, slot = pid[ok], slot[ok]                                 # the tokens that are there
    total = total.transpose(1, 2)[ok]                             # [tokens, H]
    new = (t >= x["first_pos"][:, None])[ok]
    old = st["weights"][pid, :, slot]
    if case["decay"] == 0.0:
        old = torch.zeros_like(old)
    old = torch.where(new[:, None], 0.0, old * case["decay"])
    st["weights"][pid, :, slot] = old + total


def _evict_plain(st):
    case, x, routes = st["case"], st["x"], st["routes"]
    B, H = case["seqs"], case["kv_heads"]
    begin = x["seq_route_begin"].long()
    # (the last route is the empty one, the one before it holds the last tokens)
    x["held"] = x["routes"][begin[1:] - 2, 3]
    held, keep = x["held"].long(), x["keep"].long()
    pid, slot, ok = _places(st)
    T = pid.shape[1]
    t = torch.arange(T, device=DEVICE)
    kept = torch.minimum(held, keep)
    first = torch.clamp(kept, max=case["first"])
    last = torch.clamp(kept - first, max=case["last"])
    w = x["weights"][pid, :, slot].transpose(1, 2).contiguous()   # [B, H, T]
    stays = (t < first[:, None]) | (t >= (held - last)[:, None])
    w = torch.where(stays[:, None], math.inf, w)
    w = torch.where(ok[:, None], w, -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    most = int(case["keep"])
    order = order[..., :most] if T >= most else order
    rank = torch.arange(order.shape[-1], device=DEVICE)
    order = torch.where(rank < kept[:, None, None], order, T)
    order = torch.sort(order, dim=-1).values                      # [B, H, n]: kept, in order
    real = rank < kept[:, None]                                   # [B, n]
    src = order.clamp(max=T - 1).transpose(1, 2)                  # [B, n, H]
    b = torch.arange(B, device=DEVICE)[:, None]
    spid, sslot = pid[b[..., None], src], slot[b[..., None], src]
    into = x["into"].long()
    at = (routes[into, 4].long()[:, None] + rank // PAGE)
    dpid = x["page_ids"][at.clamp(max=x["page_ids"].numel() - 1)].long()
    dpid, dslot = dpid[real], (rank % PAGE).expand(B, -1)[real]   # [tokens]
    spid, sslot = spid[real], sslot[real]                         # [tokens, H]
    h = torch.arange(H, device=DEVICE)
    for name, is_v in (("k", False), ("v", True)):
        pages = _pages(case, x[name + "_pool"])
        got = pages[spid, h, :, sslot] if is_v else pages[spid, h, sslot]     # [tokens, H, 128]
        if case["fp8"]:
            scale = x[name + "_scale"]
            was = scale[spid, h]                                  # [tokens, H]
            # a page's scale: the largest that its tokens had
            new = torch.zeros_like(scale).scatter_reduce_(
                0, dpid[:, None].expand(-1, H), was, "amax", include_self=True)
            got = _code(_decode(got) * was[..., None] / new[dpid][..., None])
            scale[dpid] = new[dpid]
        if is_v:
            pages[dpid, :, :, dslot] = got
        else:
            pages[dpid, :, dslot] = got
    x["weights"][dpid, :, dslot] = x["weights"][spid, h, sslot]
    # the other routes of the sequences are empty now
    routes[:, 3] = routes[:, 2]
    routes[into, 3] += kept.int()


# --------------------------------------------------------------------- work
def _seen(p, sinks, window):
    """Tokens that a row at position p sees."""
    w = min(window, p + 1)
    return w + min(sinks, p + 1 - w)


def work(case):
    Hq, H = case["q_heads"], case["kv_heads"]
    lens = _lengths(case)
    N = sum(n for _, n in lens)
    rows, _ = _table(case)
    elem = 1 if case["fp8"] else 2
    scale = 4 / PAGE if case["fp8"] else 0      # bytes of a scale per token and KV head
    tables = 24 * len(rows) + 8 * case["seqs"]
    if case["op"] == "window":
        s, w = case["sinks"], case["window"]
        tokens = pairs = 0
        for c, n in lens:
            if n:
                lo = min(max(0, c - w + 1), c + n)                # the window's first token
                tokens += c + n - lo + min(s, lo) if w else min(s, c + n)
                pairs += sum(_seen(p, s, w) for p in range(c, c + n))
        return {"bytes": 2 * N * Hq * DIM * 2 + 4 * N * Hq + tables + tokens / 4
                + 2 * tokens * H * (DIM * elem + scale), "flops": 4 * pairs * Hq * DIM}
    if case["op"] == "weights":
        tokens = sum(c + n for c, n in lens if n)
        old = tokens - N if case["decay"] != 0.0 else 0
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in lens)
        return {"bytes": N * Hq * (2 * DIM + 4) + tables + tokens / 4
                + tokens * H * (DIM * elem + scale + 4) + old * H * 4, "flops": 2 * pairs * Hq * DIM}
    held = sum(c for c, _ in lens)
    kept = sum(min(c, case["keep"]) for c, _ in lens)
    return {"bytes": tables + held / 4 + 4 * held * H + kept * H * (2 * 2 * DIM * elem + 4 + 4 * scale),
            "flops": 0}


# -------------------------------------------------------------------- exact
def _exact_kv(case, x, rows, g, want_v):
    """K (and V) [tokens, 128] of KV head g of the routes in rows, 64 bits."""
    out = []
    for name in ("k", "v") if want_v else ("k",):
        parts = [torch.empty((0, DIM), device=DEVICE, dtype=torch.float64)]
        for _, _, t0, t1, base, _ in rows:
            n = t1 - t0
            ids = x["page_ids"][base:base + -(-n // PAGE)].long()
            y = _pages(case, x[name + "_pool"])[ids, g]
            y = _decode(y).double() * x[name + "_scale"][ids, g].double()[:, None, None] \
                if case["fp8"] else y.double()
            if name == "v":
                y = y.transpose(1, 2)
            parts.append(y.reshape(-1, DIM)[:n])
        out.append(torch.cat(parts))
    return out


def _exact_window(case, x):
    rows, begin = _table(case)
    H, G = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    N = x["q"].shape[0]
    out = torch.zeros((N, H, G, DIM), device=DEVICE, dtype=torch.float64)
    lse = torch.full((N, H, G), -math.inf, device=DEVICE, dtype=torch.float64)
    at = 0
    for b, (c, n) in enumerate(_lengths(case)):
        for g in range(H):
            k, v = _exact_kv(case, x, rows[begin[b]:begin[b + 1]], g, True)
            for i0 in range(0, n, 4096):
                i1 = min(n, i0 + 4096)
                q = x["q"][at + i0:at + i1].view(i1 - i0, H, G, DIM)[:, g].double()
                s = torch.matmul(q.reshape(-1, DIM), k.t().contiguous()) * SCALE
                s = s.view(i1 - i0, G, -1)
                back = (c + torch.arange(i0, i1, device=DEVICE))[:, None] - \
                    torch.arange(c + n, device=DEVICE)            # how far behind the row
                far = (back >= case["window"]) & \
                    (torch.arange(c + n, device=DEVICE) >= case["sinks"])
                s.masked_fill_(((back < 0) | far)[:, None, :], -math.inf)
                z = torch.logsumexp(s, -1)
                lse[at + i0:at + i1, g] = z
                p = torch.exp(s - z[:, :, None]).view(-1, s.shape[-1])
                p = torch.nan_to_num(p)                           # a row that sees nothing
                out[at + i0:at + i1, g] = torch.matmul(p, v).view(i1 - i0, G, DIM)
        at += n
    return {"out": out.reshape(N, -1, DIM), "lse": lse.reshape(N, -1)}


def _exact_weights(case, x):
    rows, begin = _table(case)
    H, G = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    got = x["weights"].double()
    at = 0
    for b, (c, n) in enumerate(_lengths(case)):
        mine = rows[begin[b]:begin[b + 1]]
        place = torch.cat([x["page_ids"][base + torch.arange(t1 - t0, device=DEVICE) // PAGE].long()
                           * PAGE + torch.arange(t1 - t0, device=DEVICE) % PAGE
                           for _, _, t0, t1, base, _ in mine])
        for g in range(H):
            (k,) = _exact_kv(case, x, mine, g, False)
            total = torch.zeros(c + n, device=DEVICE, dtype=torch.float64)
            for i0 in range(0, n, 2048):
                i1 = min(n, i0 + 2048)
                q = x["q"][at + i0:at + i1].view(i1 - i0, H, G, DIM)[:, g].double()
                s = torch.matmul(q.reshape(-1, DIM), k.t().contiguous()).view(i1 - i0, G, -1) * SCALE
                z = x["lse"][at + i0:at + i1].view(i1 - i0, H, G)[:, g].double()
                e = torch.exp(s - z[:, :, None])
                hide = torch.arange(c + n, device=DEVICE) > \
                    (c + torch.arange(i0, i1, device=DEVICE))[:, None]
                total += e.masked_fill_(hide[:, None, :], 0.0).sum((0, 1))
            old = got[place // PAGE, g, place % PAGE] * case["decay"]
            old[c:] = 0.0
            got[place // PAGE, g, place % PAGE] = old + total
        at += n
    return {"weights": got}


def _exact_evict(case, x):
    """Sequence by sequence and head by head: whole numbers, copies, and codes."""
    rows, begin = _table(case)
    H = case["kv_heads"]
    ends = [list(r) for r in rows]
    pools = {n: _pages(case, x[n + "_pool"]) for n in ("k", "v")}
    for b, (c, _) in enumerate(_lengths(case)):
        mine, dst = rows[begin[b]:begin[b + 1] - 1], begin[b + 1] - 1
        page = torch.cat([x["page_ids"][base + torch.arange(t1 - t0, device=DEVICE) // PAGE].long()
                          for _, _, t0, t1, base, _ in mine])
        slot = torch.cat([torch.arange(t1 - t0, device=DEVICE) % PAGE for _, _, t0, t1, _, _ in mine])
        n = min(c, case["keep"])
        first = min(n, case["first"])
        last = min(n - first, case["last"])
        for r in range(begin[b], dst):
            ends[r][3] = ends[r][2]
        ends[dst][3] = ends[dst][2] + n
        to = torch.arange(n, device=DEVICE)
        dpage, dslot = x["page_ids"][rows[dst][4] + to // PAGE].long(), to % PAGE
        for g in range(H):
            w = x["weights"][page, g, slot].double()
            mid = torch.arange(first, c - last, device=DEVICE)
            by = torch.argsort(w[mid], descending=True, stable=True)[:n - first - last]
            idx = torch.cat((torch.arange(first, device=DEVICE), mid[by].sort().values,
                             torch.arange(c - last, c, device=DEVICE)))
            sp, ss = page[idx], slot[idx]
            for name, is_v in (("k", False), ("v", True)):
                pool = pools[name]
                y = pool[sp, g, :, ss] if is_v else pool[sp, g, ss]           # [n, 128]
                if case["fp8"]:
                    scale = x[name + "_scale"]
                    was = scale[sp, g]
                    new = torch.stack([z.max() for z in was.split(PAGE)])
                    scale[dpage[::PAGE], g] = new
                    near = _decode(y).double() * was.double()[:, None] / \
                        new.double()[to // PAGE][:, None]
                    # (64 bits to E4M3 at once: 32 would round twice)
                    y = _nearest_code(near)
                if is_v:
                    pool[dpage, g, :, dslot] = y
                else:
                    pool[dpage, g, dslot] = y
            x["weights"][dpage, g, dslot] = x["weights"][sp, g, ss]
    got = {"routes": torch.tensor(ends, dtype=torch.int32, device=DEVICE), "k_pool": x["k_pool"],
           "v_pool": x["v_pool"], "weights": x["weights"]}
    if case["fp8"]:
        got.update(k_pool=x["k_pool"].view(torch.float8_e4m3fn),
                   v_pool=x["v_pool"].view(torch.float8_e4m3fn),
                   k_scale=x["k_scale"], v_scale=x["v_scale"])
    return got


def _nearest_code(x):
    """E4M3 codes of 64-bit values up to 448 in size, round to nearest even."""
    a = x.abs()
    exp = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    step = torch.exp2(exp - 3)
    return _code(torch.copysign(torch.round(a / step) * step, x).float())


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "evict":
        # a launch for each sequence, head and page
        if case["seqs"] * case["kv_heads"] * (40 + case["keep"] / PAGE) > 1 << 18:
            return None
        return _exact_evict(case, x)
    return _exact_window(case, x) if case["op"] == "window" else _exact_weights(case, x)
