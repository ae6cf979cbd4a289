"""The operators on whole rows of tokens that this library's speed is measured on.

One case is one call of one operator for one attention layer:

* ``prompt``  causal attention of packed prompts over their paged cache
  (``kf.prompt_attn``): sequence b has ``rows`` query rows behind ``ctx`` cached
  tokens; row i sits at position ctx + i and sees the tokens up to itself;
* ``tree``    attention of drafted trees over the cache (``kf.tree_attn``): each
  sequence drafts ``rows`` tokens (a random tree), every one sees the whole
  cache of ``ctx`` tokens and its own ancestors;
* ``append``  rows of K/V written into the cache (``kf.kv_append_rows``): ``rows``
  per sequence behind ``ctx`` resident tokens, picked from ``pool_rows`` times as
  many drafted ones through a list where ``pool_rows`` > 1.

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


def _case(name, op, seqs, q_heads, kv_heads, rows, ctx, part, *, fp8=False, head_major=False,
          permuted=False, pool_rows=1, lens=1):
    return {"name": name, "op": op, "seqs": seqs, "q_heads": q_heads, "kv_heads": kv_heads,
            "rows_lo": rows[0], "rows_hi": rows[1], "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "part": part, "fp8": fp8, "head_major": head_major, "permuted": permuted,
            "pool_rows": pool_rows, "lens": lens}


def listed():
    return [
        # the smallest prompt: one short question on a small layer, latency only
        _case("prompt_short", "prompt", 1, 8, 2, (37, 37), (0, 0), 2048),
        # a batch of chat prompts of different lengths on a Llama-3.1-8B layer
        _case("prompt_pack", "prompt", 16, 32, 8, (100, 2000), (0, 0), 8192, permuted=True),
        # multi-head attention (one query head per KV head), head-major pools
        _case("prompt_mha", "prompt", 4, 32, 32, (700, 1500), (0, 0), 8192, head_major=True),
        # chunked prefill: 512 rows of each request behind 32K cached tokens, fp8, 64/8 heads
        _case("prompt_chunk_fp8", "prompt", 4, 64, 8, (512, 512), (32768, 32768), 16384, fp8=True,
              permuted=True),
        # one long document, 16K tokens
        _case("prompt_long", "prompt", 1, 32, 8, (16384, 16384), (0, 0), 8192),
        # the smallest tree: five drafted tokens of one chat
        _case("tree_tiny", "tree", 1, 8, 2, (5, 5), (700, 700), 2048),
        # agentic serving: 4 to 12 drafted tokens over 2K .. 64K in one permuted pool
        _case("tree_agentic", "tree", 48, 32, 8, (4, 12), (2048, 65536), 16384, permuted=True),
        # a Llama-3.1-8B layer at 32K tokens, 32 drafted tokens per sequence
        _case("tree_llama", "tree", 16, 32, 8, (32, 32), (32768, 32768), 8192),
        # a 70B-like layer (64/8 heads) with fp8 K/V at 64K tokens, 16 drafted tokens
        _case("tree_fp8", "tree", 32, 64, 8, (16, 16), (65536, 65536), 16384, fp8=True),
        # the accepted paths of 16 trees of 32 tokens: 1 to 6 rows each, through a list
        _case("append_accept", "append", 16, 32, 8, (1, 6), (500, 3000), 8192, permuted=True,
              pool_rows=6),
        # the K/V of chat prompts written into fp8 pages
        _case("append_pack_fp8", "append", 32, 64, 8, (100, 4000), (0, 40), 8192, fp8=True,
              permuted=True),
        # the K/V of a 16K document written into two routes
        _case("append_long", "append", 1, 32, 8, (16384, 16384), (0, 0), 8192),
    ]


_HEADS = ((8, 2), (16, 2), (32, 8), (64, 8), (32, 32), (40, 8), (24, 8), (64, 4), (8, 1), (16, 16))


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {op: max(_cost(work(c)) for c in listed() if c["op"] == op)
            for op in ("prompt", "tree", "append")}
    while True:
        op = rng.choice(("prompt", "tree", "append"))
        q_heads, kv_heads = rng.choice(_HEADS)
        lo = spread(1, {"prompt": 4000, "tree": 64, "append": 8000}[op])
        hi = lo if rng.random() < 0.3 else min(16384, spread(lo, 20 * lo))
        clo = spread(1, 60000) if op == "tree" or rng.random() < 0.4 else 0
        chi = clo if rng.random() < 0.3 else min(65536, spread(max(1, clo), 20 * max(1, clo)))
        if op == "tree":
            hi = min(64, hi)
        elif op == "append":
            clo, chi = clo % 100, chi % 100
        c = _case("", op, spread(1, 64), q_heads, kv_heads, (min(lo, hi), hi),
                  (min(clo, chi), chi), rng.choice((2048, 4096, 8192, 16384)),
                  fp8=rng.random() < 0.35, head_major=rng.random() < 0.25,
                  permuted=rng.random() < 0.6,
                  pool_rows=rng.choice((1, 4)) if op == "append" and hi < 100 else 1,
                  lens=rng.randrange(1 << 20))
        del c["name"]
        # the padded plain forms hold every sequence at the longest one's length
        n, t = _longest(c)
        if c["seqs"] * t * kv_heads > 1 << 25 or c["seqs"] * q_heads * n * t > 9e9:
            continue
        if 2e5 <= _cost(work(c)) <= most[op]:
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
    """The most rows of a sequence, and the most tokens that its rows may see."""
    lens = _lengths(case)
    return (max(n for _, n in lens),
            max(c + n if case["op"] == "prompt" else c for c, n in lens))


def _table(case):
    """Route rows [seq, part, tok_begin, tok_end, page_base, page_cap], the CSR
    rows of the sequences, and per route the rows that an append gives it."""
    rows, begin, takes, base = [], [0], [], 0
    for b, (c, n) in enumerate(_lengths(case)):
        held = c + n if case["op"] == "prompt" else c     # resident before the call
        end = c if case["op"] == "tree" else c + n        # resident after it
        for k, t0 in enumerate(range(0, max(end, 1), case["part"])):
            t1 = min(t0 + case["part"], end)
            cap = -(-(t1 - t0) // PAGE)
            t = min(t1, max(t0, held))
            rows.append([b, k, t0, t, base, cap])
            takes.append(t1 - t)
            base += cap
        begin.append(len(rows))
    return rows, begin, takes


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


def _tree(n, rng):
    """Ancestor bits (itself among them) of each of n drafted tokens of a random tree."""
    bits = []
    for i in range(n):
        up = bits[rng.randrange(max(0, i - 6), i)] if i and rng.random() < 0.9 else 0
        b = up | 1 << i
        bits.append(b)
    return [b - (1 << 64) if b >> 63 else b for b in bits]


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
    rng = random.Random(seed)
    rows, begin, takes = _table(case)
    lens = _lengths(case)
    B, Hq, H = case["seqs"], case["q_heads"], case["kv_heads"]
    N = sum(n for _, n in lens)

    def ints(v, dtype=torch.int32):
        return torch.tensor(v, dtype=dtype, device=DEVICE)

    def normal(*size):
        return torch.randn(size, generator=gen, device=DEVICE, dtype=torch.bfloat16)

    x = {"routes": ints(rows), "seq_route_begin": ints(begin)}
    x["page_ids"], P = _page_ids(case, [r[5] for r in rows], gen)
    x["k_pool"], x["k_scale"] = _pool(case, P, (PAGE, DIM), gen)
    x["v_pool"], x["v_scale"] = _pool(case, P, (DIM, PAGE), gen)
    if case["op"] == "append":
        x["k_rows"], x["v_rows"] = (normal(N * case["pool_rows"], H, DIM) for _ in range(2))
        x["route_entry_begin"] = ints(_csr(takes))
        if case["pool_rows"] > 1:
            # an accepted path: increasing places among the sequence's drafted rows
            picks, first = [], 0
            for _, n in lens:
                picks += sorted(rng.sample(range(first, first + n * case["pool_rows"]), n))
                first += n * case["pool_rows"]
            x["row_list"] = ints(picks)
        return x
    x["q"] = normal(N, Hq, DIM)
    row_begin = _csr([n for _, n in lens])
    x["seq_row_begin"] = ints(row_begin)
    if case["op"] == "prompt":
        x["first_pos"] = ints([c for c, _ in lens])
    else:
        x["k_draft"], x["v_draft"] = normal(N, H, DIM), normal(N, H, DIM)
        x["tree_mask"] = ints([m for _, n in lens for m in _tree(n, rng)], torch.int64)
    # an attention sink: the first token of each sequence with a cache scores about 7
    # for the first row's heads
    at = [(b, rows[begin[b]][4]) for b in range(B) if rows[begin[b]][5] > 0]
    if at:
        first = x["page_ids"][ints([p for _, p in at], torch.int64)].long()
        q = x["q"][ints([row_begin[b] for b, _ in at], torch.int64)]
        sink = 0.6 * q.view(len(at), H, Hq // H, DIM).float().sum(2)
        pages = _pages(case, x["k_pool"])
        if case["fp8"]:
            pages[first, :, 0] = _code(sink / x["k_scale"][first][:, :, None])
        else:
            pages[first, :, 0] = sink.to(torch.bfloat16)
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    st = {"case": dict(case), "x": x, "err": torch.zeros(1, dtype=torch.int32, device=DEVICE),
          "most_pages": max(r[5] for r in _table(case)[0])}
    if case["op"] == "append":
        st["routes"] = x["routes"].clone()
    else:
        N, Hq = x["q"].shape[:2]
        st["longest"] = _longest(case)
        st["out"] = torch.empty((N, Hq, DIM), device=DEVICE, dtype=torch.bfloat16)
        st["lse"] = torch.empty((N, Hq), device=DEVICE)
    return st


# ---------------------------------------------------------------------- run
def run(st):
    op = st["case"]["op"]
    if op == "append":
        st["routes"].copy_(st["x"]["routes"])   # the step's route table
        if own:
            _call(st)()
        else:
            _append_plain(st)
        x = st["x"]
        got = {"routes": st["routes"], "k_pool": x["k_pool"], "v_pool": x["v_pool"]}
        if st["case"]["fp8"]:
            got.update(k_pool=x["k_pool"].view(torch.float8_e4m3fn),
                       v_pool=x["v_pool"].view(torch.float8_e4m3fn),
                       k_scale=x["k_scale"], v_scale=x["v_scale"])
        return got
    if own:
        _call(st)()
    else:
        _attend_plain(st)
    return {"out": st["out"], "lse": st["lse"]}


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
        scales = {"k_scale": x["k_scale"], "v_scale": x["v_scale"]}
        if case["op"] == "append":
            st["call"] = kf.bind_kv_append_rows(
                shape, x["k_pool"], x["v_pool"], x["k_rows"], x["v_rows"], st["routes"],
                x["route_entry_begin"], x["page_ids"], st["err"], row_list=x.get("row_list"),
                **scales)
        else:
            ws = kf.alloc_rows_workspace(shape, x["q"].shape[0], DEVICE)
            cache = (x["k_pool"], x["v_pool"], x["routes"], st["most_pages"], x["page_ids"],
                     x["seq_route_begin"], x["seq_row_begin"])
            if case["op"] == "prompt":
                st["call"] = kf.bind_prompt_attn(shape, x["q"], x["first_pos"], *cache, st["out"],
                                                 st["lse"], ws, st["err"], **scales)
            else:
                st["call"] = kf.bind_tree_attn(shape, x["q"], x["k_draft"], x["v_draft"],
                                               x["tree_mask"], *cache, st["out"], st["lse"], ws,
                                               st["err"], **scales)
    return st["call"]


def _padded(st):
    """K and V [B, H, T, 128] of every sequence's first T tokens, T the longest's
    (zeros behind a sequence's last), and the tokens each one holds."""
    case, x = st["case"], st["x"]
    H, T = case["kv_heads"], max(1, st["longest"][1])
    begin = x["seq_route_begin"].long()
    t = torch.arange(T, device=DEVICE)
    r = torch.minimum(begin[:-1, None] + t // case["part"], begin[1:, None] - 1)
    held = x["routes"][begin[1:] - 1, 3]
    ok = t < held[:, None]
    j = torch.where(ok, t - x["routes"][r, 2], 0)
    at = x["routes"][r, 4].long() + j // PAGE
    pid = torch.where(ok, x["page_ids"][at.clamp(max=x["page_ids"].numel() - 1)], 0).long()
    slot = j % PAGE
    k = _pages(case, x["k_pool"])[pid, :, slot]              # [B, T, H, 128]
    v = _pages(case, x["v_pool"])[pid, :, :, slot]
    k, v = (_decode(k), _decode(v)) if case["fp8"] else (k.float(), v.float())
    if case["fp8"]:
        k *= x["k_scale"][pid][..., None]
        v *= x["v_scale"][pid][..., None]
    return (k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous(), held)


def _attend_plain(st):
    case, x = st["case"], st["x"]
    B, Hq, H, n = case["seqs"], case["q_heads"], case["kv_heads"], st["longest"][0]
    G = Hq // H
    begin = x["seq_row_begin"].long()
    i = torch.arange(n, device=DEVICE)
    row = begin[:-1, None] + i                               # [B, n]
    real = row < begin[1:, None]
    row = torch.where(real, row, 0)
    q = x["q"][row].float().view(B, n, H, G, DIM).permute(0, 2, 3, 1, 4).reshape(B, H, G * n, DIM)
    k, v, held = _padded(st)
    t = torch.arange(k.shape[2], device=DEVICE)
    sees = (t < held[:, None])[:, None, :]                   # [B, 1 or n, T]
    if case["op"] == "prompt":
        sees = sees & (t <= (x["first_pos"][:, None] + i)[:, :, None])
    else:                                                    # the drafted tokens follow
        k = torch.cat((k, x["k_draft"][row].float().transpose(1, 2)), 2)
        v = torch.cat((v, x["v_draft"][row].float().transpose(1, 2)), 2)
        drafted = (x["tree_mask"][row][:, :, None] >> i & 1).bool() & real[:, None, :]
        sees = torch.cat((sees.expand(B, n, -1), drafted), 2)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(SCALE)
    s = s.view(B, H, G, n, -1).masked_fill_(~sees[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_(min=-1e30)
    total = s.sub_(top).exp_().sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, H, G * n, -1), v).view(B, H, G, n, DIM) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, Hq, DIM)
    lse = lse.permute(0, 3, 1, 2).reshape(B, n, Hq)
    # the rows of the packed outputs: place e is row e - begin[b] of sequence b
    e = torch.arange(x["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(begin, e, right=True) - 1
    st["out"].copy_(o[b, e - begin[b]])
    st["lse"].copy_(lse[b, e - begin[b]])


def _append_plain(st):
    case, x, routes = st["case"], st["x"], st["routes"]
    begin = x["route_entry_begin"].long()
    N = x["k_rows"].shape[0] // case["pool_rows"]
    e = torch.arange(N, device=DEVICE)
    r = torch.searchsorted(begin, e, right=True) - 1
    j = (routes[r, 3] - routes[r, 2]) + e - begin[r]
    pid = x["page_ids"][routes[r, 4].long() + j // PAGE].long()
    slot = j % PAGE
    src = x["row_list"].long() if "row_list" in x else e
    for pool, scale, rows, is_v in ((x["k_pool"], x["k_scale"], x["k_rows"][src], False),
                                    (x["v_pool"], x["v_scale"], x["v_rows"][src], True)):
        pages = _pages(case, pool)
        if case["fp8"]:
            # slot after slot: the token at slot 0 sets its page's scale to amax/28; a
            # later one beyond 448 * scale re-encodes the slots before it to amax/28
            tok = rows.float()
            amax = tok.abs().amax(-1)
            fresh = amax / torch.full_like(amax, 28.0)
            fresh = torch.where(amax > 0, fresh, torch.ones_like(fresh))
            for s in range(PAGE):
                now = (slot == s).nonzero().squeeze(1)
                p, f, old = pid[now], fresh[now], scale[pid[now]]
                if s == 0:
                    new = f
                else:
                    over = amax[now] > 448.0 * old
                    new = torch.where(over, f, old)
                    held = pages[p, :, :, :s] if is_v else pages[p, :, :s]
                    redone = _code(_decode(held) * old[..., None, None] / new[..., None, None])
                    held = torch.where(over[..., None, None], redone, held)
                    if is_v:
                        pages[p, :, :, :s] = held
                    else:
                        pages[p, :, :s] = held
                scale[p] = new
                code = _code(tok[now] / new[..., None])
                if is_v:
                    pages[p, :, :, s] = code
                else:
                    pages[p, :, s] = code
        elif is_v:
            pages[pid, :, :, slot] = rows
        else:
            pages[pid, :, slot] = rows
    routes[:, 3] += (begin[1:] - begin[:-1]).int()


# --------------------------------------------------------------------- work
def work(case):
    Hq, H = case["q_heads"], case["kv_heads"]
    lens = _lengths(case)
    N = sum(n for _, n in lens)
    rows, _, _ = _table(case)
    elem = 1 if case["fp8"] else 2
    scale = 8 / PAGE if case["fp8"] else 0      # bytes of scales per token and KV head
    tables = 24 * len(rows) + 8 * case["seqs"]
    if case["op"] == "append":
        return {"bytes": N * H * (2 * DIM * (2 + elem) + scale) + 4 * N / PAGE + tables, "flops": 0}
    data = 2 * N * Hq * DIM * 2 + N * Hq * 4 + tables
    if case["op"] == "prompt":
        tokens = sum(c + n for c, n in lens)
        pairs = sum(n * c + n * (n + 1) // 2 for c, n in lens)
    else:
        tokens = sum(c for c, _ in lens)
        pairs = sum(n * (c + min(n, 6)) for c, n in lens)
        data += N * H * 2 * DIM * 2 + 8 * N
    return {"bytes": data + tokens * H * (2 * DIM * elem + scale) + tokens / 4,
            "flops": 4 * pairs * Hq * DIM}


# -------------------------------------------------------------------- exact
def _exact_kv(case, x, rows, g, tokens):
    """K and V [tokens, 128] of KV head g of the routes in rows, 64 bits."""
    ks, vs = [], []
    for _, _, t0, t1, base, _ in rows:
        n = min(t1, tokens) - t0
        if n <= 0:
            continue
        ids = x["page_ids"][base:base + -(-n // PAGE)].long()
        k, v = _pages(case, x["k_pool"])[ids, g], _pages(case, x["v_pool"])[ids, g]
        if case["fp8"]:
            k, v = _decode(k), _decode(v)
        k, v = k.double(), v.double()
        if case["fp8"]:
            k *= x["k_scale"][ids, g].double()[:, None, None]
            v *= x["v_scale"][ids, g].double()[:, None, None]
        ks.append(k.reshape(-1, DIM)[:n])
        vs.append(v.transpose(1, 2).reshape(-1, DIM)[:n])
    none = torch.empty((0, DIM), device=DEVICE, dtype=torch.float64)
    return torch.cat([none] + ks), torch.cat([none] + vs)


def _exact_attention(case, x):
    rows, begin, _ = _table(case)
    H, G = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    N = x["q"].shape[0]
    out = torch.zeros((N, H, G, DIM), device=DEVICE, dtype=torch.float64)
    lse = torch.full((N, H, G), -math.inf, device=DEVICE, dtype=torch.float64)
    at = 0
    for b, (c, n) in enumerate(_lengths(case)):
        mine = rows[begin[b]:begin[b + 1]]
        for g in range(H):
            k, v = _exact_kv(case, x, mine, g, 1 << 30)
            if case["op"] == "tree":
                k = torch.cat((k, x["k_draft"][at:at + n, g].double()))
                v = torch.cat((v, x["v_draft"][at:at + n, g].double()))
            for i0 in range(0, n, 4096):
                i1 = min(n, i0 + 4096)
                q = x["q"][at + i0:at + i1].view(i1 - i0, H, G, DIM)[:, g].double()
                s = torch.matmul(q.reshape(-1, DIM), k.t().contiguous()) * SCALE
                s = s.view(i1 - i0, G, -1)
                place = torch.arange(i0, i1, device=DEVICE)
                if case["op"] == "prompt":
                    hide = torch.arange(c + n, device=DEVICE) > (c + place)[:, None]
                else:
                    bits = x["tree_mask"][at + i0:at + i1]
                    seen = torch.stack([(bits >> j) & 1 for j in range(n)], 1) == 1
                    cached = torch.ones((i1 - i0, c), dtype=torch.bool, device=DEVICE)
                    hide = ~torch.cat((cached, seen), 1)
                s.masked_fill_(hide[:, None, :], -math.inf)
                z = torch.logsumexp(s, -1)
                lse[at + i0:at + i1, g] = z
                p = torch.exp(s - z[:, :, None]).view(-1, s.shape[-1])
                out[at + i0:at + i1, g] = torch.matmul(p, v).view(i1 - i0, G, DIM)
        at += n
    return {"out": out.reshape(N, -1, DIM), "lse": lse.reshape(N, -1)}


def _exact_append(case, x):
    """Page by page: whole numbers and codes, so only the scales are computed values."""
    rows, _, takes = _table(case)
    ends, src, dst, at = [], [], [], 0
    for (b, k, t0, t1, base, cap), n in zip(rows, takes):
        dst += [(base, t1 - t0 + i) for i in range(n)]
        src += list(range(at, at + n))
        at += n
        ends.append([b, k, t0, t1 + n, base, cap])
    routes = torch.tensor(ends, dtype=torch.int32, device=DEVICE)
    if "row_list" in x:
        src = x["row_list"].tolist()
    place = torch.tensor([p + j // PAGE for p, j in dst], device=DEVICE)
    page, slot = x["page_ids"][place].long(), torch.tensor([j % PAGE for _, j in dst], device=DEVICE)
    got = {"routes": routes}
    for name, is_v in (("k", False), ("v", True)):
        new = x[name + "_rows"][torch.tensor(src, device=DEVICE)]
        pool = _pages(case, x[name + "_pool"])
        flat = (pool.transpose(2, 3) if is_v else pool)      # a view [P, H, 16, 128]
        if case["fp8"]:
            scale = x[name + "_scale"]
            big = new.float().abs().amax(-1)
            opens = slot == 0
            scale[page[opens]] = (big[opens].double() / 28.0).float()
            mine = scale[page]
            if bool((big > 448.0 * mine).any()):
                return None                                  # a page would be re-encoded
            new = _code(new.float() / mine[..., None])
            got[name + "_scale"] = scale
        flat[page, :, slot] = new
        got[name + "_pool"] = (x[name + "_pool"].view(torch.float8_e4m3fn) if case["fp8"]
                               else x[name + "_pool"])
    return got


def exact(case, seed):
    x = _inputs(case, seed)
    return _exact_append(case, x) if case["op"] == "append" else _exact_attention(case, x)
