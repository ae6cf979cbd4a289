"""Calls of the operators that keep a cache within a budget (window attention,
attention weights, eviction) on the GPU, and their comparison against the fp64
oracle.  Caches and rows are rows_testlib's."""
from __future__ import annotations

import numpy as np

import oracle
from rows_testlib import DIM, PAGE, SCALE, Cache, Rows  # noqa: F401


def _dev(x):
    from paper_2606_29207_amd.step import _to_dev
    return _to_dev(x, "cuda")


def _wide(x, pad):
    """Rows as parts of wider ones."""
    import torch
    t = _dev(x)
    if not pad:
        return t
    w = torch.full((t.shape[0], t.shape[1] * DIM + pad), float("nan"), dtype=torch.bfloat16,
                   device="cuda")
    w[:, :t.shape[1] * DIM] = t.reshape(t.shape[0], -1)
    return w[:, :t.shape[1] * DIM].unflatten(1, (t.shape[1], DIM))


# ------------------------------------------------------------------- window
def window_oracle(r, sinks, window, scale=SCALE):
    c = r.cache
    return oracle.rows_attn(r.q, r.row_begin, c.k_pool, c.v_pool, c.routes, c.page_ids,
                            c.seq_route_begin, num_kv_heads=c.H, scale=scale,
                            max_pages_per_route=c.max_pages, first_pos=r.first_pos,
                            k_scale=c.k_scale, v_scale=c.v_scale, sinks=sinks, window=window)


def window_gpu(r, sinks, window, scale=SCALE, head_major=False, pad=0, stream=None, d=None,
               run=True):
    """Outputs (numpy, float64) and flags of kf_window_attn."""
    import torch
    from paper_2606_29207_amd import kf
    c = r.cache
    d = c.device(head_major) if d is None else d
    q = _wide(r.q, pad)
    N, Hq = q.shape[:2]
    shape = c.shape(Hq, scale, head_major)
    out = torch.full((N, Hq, DIM), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((N, Hq), float("nan"), device="cuda")
    ws = kf.alloc_rows_workspace(shape, N)
    ws.fill_(0xFF)
    call = kf.bind_window_attn(shape, q, _dev(r.first_pos), sinks, window, d["k_pool"], d["v_pool"],
                               d["routes"], c.max_pages, d["page_ids"], d["seq_route_begin"],
                               _dev(r.row_begin), out, lse, ws, d["err"], k_scale=d["k_scale"],
                               v_scale=d["v_scale"])
    if not run:
        return call, out, lse, d["err"]
    if stream is not None:
        torch.cuda.synchronize()
    call(stream)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy(), int(d["err"].item())


# ------------------------------------------------------------------ weights
def rows_lse(r, scale=SCALE):
    """The rows' lse, as their attention would return it."""
    return r.oracle(scale)[1].astype(np.float32)


def start_weights(c, seed=0):
    """Weights of every slot of a pool, those that hold no token included."""
    rng = np.random.default_rng(seed)
    return (rng.random((c.k_pool.shape[0], c.H, PAGE)) ** 4 * 3).astype(np.float32)


def weights_oracle(r, lse, weights, decay, scale=SCALE):
    c = r.cache
    return oracle.attn_weights(r.q, lse, r.row_begin, r.first_pos, c.k_pool, c.routes, c.page_ids,
                               weights, num_kv_heads=c.H, scale=scale, decay=decay,
                               max_pages_per_route=c.max_pages, k_scale=c.k_scale)


def weights_gpu(r, lse, weights, decay, scale=SCALE, head_major=False, pad=0, stream=None, d=None,
                run=True):
    """The new weights (numpy float32) and flags of kf_attn_weights."""
    import torch
    from paper_2606_29207_amd import kf
    c = r.cache
    d = c.device(head_major) if d is None else d
    q = _wide(r.q, pad)
    w = _dev(weights)
    call = kf.bind_attn_weights(c.shape(q.shape[1], scale, head_major), q, _dev(lse),
                                _dev(r.first_pos), d["k_pool"], d["routes"], c.max_pages,
                                d["page_ids"], _dev(r.row_begin), decay, w, d["err"],
                                k_scale=d["k_scale"])
    if not run:
        return call, w, d["err"]
    if stream is not None:
        torch.cuda.synchronize()
    call(stream)
    torch.cuda.synchronize()
    return w.cpu().numpy(), int(d["err"].item())


def weights_segments(r, chunk_pages=16):
    """How many workgroups share the columns of the same keys, from the workspace that the
    launch asks for: 256 sums of each, for stretches of chunk_pages pages."""
    from paper_2606_29207_amd import kf
    c = r.cache
    n, R = kf.attn_weights_workspace_bytes(c.shape(r.q.shape[1]), r.q.shape[0], len(c.routes),
                                           c.max_pages), len(c.routes)
    chunks = -(-min(c.max_pages, len(c.page_ids)) // chunk_pages)
    return max(1, n // (R * chunks * c.H * 1024))


def assert_weights(got, ref, before, what=""):
    """Weights against the oracle's.  A term exp(s - lse) is off by what its exponent is:
    the 128 products of a score, added in 32 bits, by at most 128 x 2^-24 of the sum of
    their sizes, below 1e-4 for N(0, 1) (as lse is), and the roundings of the exponent
    and of exp2, a few 2^-24 of numbers below 2^5, well below 2e-5; a sum of n terms of
    one sign by at most n x 2^-24 of it, and the old weight by two roundings."""
    w, flags = got
    r, r_flags, terms = ref
    assert flags == r_flags, f"{what}: flags {flags} != {r_flags}"
    assert np.array_equal(np.isnan(w), np.isnan(r)), f"{what}: NaN positions differ"
    bound = (1.2e-4 + terms * 2.0 ** -24) * np.abs(r) + 2.0 ** -22 * np.abs(before) + 1e-30
    fine = np.isfinite(r)
    over = (np.abs(w.astype(np.float64) - r) - bound)[fine]
    assert over.size == 0 or over.max() <= 0, f"{what}: weights beyond their bound by {over.max():.3e}"


# -------------------------------------------------------------------- evict
class Evictable(Cache):
    """A cache whose sequences end in an empty route of `room[b]` pages (by default
    what keep[b] tokens take)."""

    def __init__(self, lens, keep, *, room=None, dst_begin=0, junk=True, **kw):
        super().__init__(lens, extra_pages=0, **kw)
        rng = np.random.default_rng(kw.get("seed", 0) + 1000)
        self.keep = np.array(keep, np.int32)
        room = [-(-min(n, int(k)) // PAGE) for n, k in zip(lens, keep)] if room is None else room
        rows, begin, base = [], [0], len(self.page_ids)
        for b in range(len(lens)):
            rows += [list(r) for r in self.routes[self.seq_route_begin[b]:self.seq_route_begin[b + 1]]]
            rows.append([b, 99, dst_begin, dst_begin, base, room[b]])
            base += room[b]
            begin.append(len(rows))
        self.routes = np.array(rows, np.int32).reshape(-1, 6)
        self.seq_route_begin = np.array(begin, np.int32)
        self.into = self.seq_route_begin[1:] - 1
        old_P, old_ids = self.k_pool.shape[0], len(self.page_ids)
        P = base + 3
        perm = rng.permutation(P)
        grow = (lambda x: None if x is None else
                np.concatenate([x, np.full((P - old_P,) + x.shape[1:], x.dtype.type(
                    np.nan if x.dtype.kind == "f" else 0x7F), x.dtype)])[np.argsort(perm)])
        self.k_pool, self.v_pool, self.k_scale, self.v_scale = (
            grow(x) for x in (self.k_pool, self.v_pool, self.k_scale, self.v_scale))
        # (page p of before is perm[p] now)
        self.page_ids = perm[np.concatenate([self.page_ids, np.arange(old_P, old_P + base - old_ids)])
                             ].astype(np.int32)
        self.max_pages = int(max(self.routes[:, 5]))
        self.weights = (rng.random((P, self.H, PAGE)) ** 6).astype(np.float32)
        self.weights[rng.random(self.weights.shape) < 0.2] = 0.0


def evict_oracle(c, first, last, max_keep=None):
    return oracle.kv_evict(c.k_pool, c.v_pool, c.weights, c.routes, c.page_ids, c.seq_route_begin,
                           c.into, c.keep, max_keep=int(c.keep.max()) if max_keep is None else max_keep,
                           keep_first=first, keep_last=last, max_pages_per_route=c.max_pages,
                           k_scale=c.k_scale, v_scale=c.v_scale)


def evict_parts(c, max_keep=None, G=2):
    """Into how many parts an eviction's launch divides a sequence and KV head, from the
    workspace that it asks for: a list of max_keep places each, and for each of several
    parts 4 words and 3 x 2048 bins."""
    from paper_2606_29207_amd import kf
    max_keep = int(c.keep.max()) if max_keep is None else max_keep
    units, up = len(c.lens) * c.H, lambda x: -(-x // 256) * 256
    more = (kf.kv_evict_workspace_bytes(c.shape(c.H * G), max_keep) - up(len(c.lens) * 8) - 256
            - up(units * max_keep * 4))
    parts = more // (units * 4 * (4 + 3 * 2048))
    assert more == parts * units * 3 * 2048 * 4 + up(parts * units * 16)
    return max(1, parts)


def evict_gpu(c, first, last, max_keep=None, head_major=False, G=2, stream=None, run=True, d=None):
    """k_pool, v_pool, weights, routes, k_scale, v_scale (numpy, as the oracle lays them
    out) and flags of kf_kv_evict."""
    import torch
    from paper_2606_29207_amd import kf
    d = c.device(head_major) if d is None else d
    w = _dev(c.weights)
    shape = c.shape(c.H * G, SCALE, head_major)
    max_keep = int(c.keep.max()) if max_keep is None else max_keep
    ws = torch.full((kf.kv_evict_workspace_bytes(shape, max_keep),), 0xFF, dtype=torch.uint8,
                    device="cuda")
    call = kf.bind_kv_evict(shape, d["k_pool"], d["v_pool"], w, d["routes"], c.max_pages,
                            d["page_ids"], d["seq_route_begin"], _dev(c.into.astype(np.int32)),
                            _dev(c.keep), max_keep, first, last, d["err"], k_scale=d["k_scale"],
                            v_scale=d["v_scale"], workspace=ws)
    if not run:
        return call, w, d
    if stream is not None:
        torch.cuda.synchronize()
    call(stream)
    torch.cuda.synchronize()
    return evict_result(c, d, w, head_major)


def evict_result(c, d, w, head_major=False):
    import torch

    def pool(t):
        t = t.transpose(0, 1) if head_major else t
        t = t.contiguous()
        return t.cpu().numpy() if c.fp8 else t.view(torch.int16).cpu().numpy().view(np.uint16)

    return (pool(d["k_pool"]), pool(d["v_pool"]), w.cpu().numpy(), d["routes"].cpu().numpy(),
            d["k_scale"].cpu().numpy() if c.fp8 else None,
            d["v_scale"].cpu().numpy() if c.fp8 else None, int(d["err"].item()))


def assert_evicted(got, ref, what=""):
    """Bit for bit: whole numbers, copies, and codes by one rule in 32 bits."""
    assert got[6] == ref[6], f"{what}: flags {got[6]} != {ref[6]}"
    for x, y, n in zip(got, ref, ("k_pool", "v_pool", "weights", "routes", "k_scale", "v_scale")):
        if y is None:
            continue
        if y.dtype.kind == "f":
            x, y = x.view(np.uint32), np.ascontiguousarray(y).view(np.uint32)
        assert np.array_equal(x, y), f"{what}: {n} differs at {np.argwhere(x != y)[:4].tolist()}"
