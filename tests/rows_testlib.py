"""Paged caches with rows of queries or drafted tokens for the tests of the row
operators: a seeded builder, the call on the GPU, and the comparison against
the fp64 oracle."""
from __future__ import annotations

import math

import numpy as np

import oracle

PAGE, DIM = 16, 128
SCALE = 1.0 / math.sqrt(DIM)


def bits(x):
    """float32 -> bf16 bits, round to nearest even (finite input)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


class Cache:
    """Sequences of lens[b] resident tokens in routes of `part` tokens, `spare`
    more pages in each sequence's last route, over a permuted pool whose unused
    slots hold NaN.  first[b]: the sequence's first token."""

    def __init__(self, lens, *, H=2, fp8=False, part=1 << 30, spare=0, seed=0, first=None,
                 extra_pages=3):
        self.H, self.fp8, self.lens = H, fp8, list(lens)
        rng = np.random.default_rng(seed)
        first = [0] * len(lens) if first is None else first
        rows, begin, base = [], [0], 0
        for b, n in enumerate(lens):
            starts = list(range(0, n, part)) or [0]
            for k, t0 in enumerate(starts):
                t1 = min(t0 + part, n)
                cap = -(-(t1 - t0) // PAGE) + (spare if t0 == starts[-1] else 0)
                rows.append([b, k, first[b] + t0, first[b] + t1, base, cap])
                base += cap
            begin.append(len(rows))
        self.routes = np.array(rows, np.int32).reshape(-1, 6)
        self.seq_route_begin = np.array(begin, np.int32)
        P = base + extra_pages
        self.page_ids = rng.permutation(P)[:base].astype(np.int32)
        self.max_pages = int(max([r[5] for r in rows], default=0))
        if fp8:
            self.k_pool = np.full((P, H, PAGE, DIM), 0x7F, np.uint8)
            self.v_pool = np.full((P, H, DIM, PAGE), 0x7F, np.uint8)
            self.k_scale = np.full((P, H), np.nan, np.float32)
            self.v_scale = np.full((P, H), np.nan, np.float32)
        else:
            self.k_pool = np.full((P, H, PAGE, DIM), 0x7FC0, np.uint16)
            self.v_pool = np.full((P, H, DIM, PAGE), 0x7FC0, np.uint16)
            self.k_scale = self.v_scale = None
        for r in rows:
            for p in range(-(-(r[3] - r[2]) // PAGE)):
                n = min(PAGE, r[3] - r[2] - p * PAGE)
                pid = self.page_ids[r[4] + p]
                k, v = (rng.standard_normal((H, n, DIM)).astype(np.float32) for _ in range(2))
                if fp8:
                    for x, scale in ((k, self.k_scale), (v, self.v_scale)):
                        s = np.abs(x).max((1, 2)) / np.float32(448)
                        scale[pid] = s
                        x /= s[:, None, None]
                    self.k_pool[pid, :, :n] = oracle.e4m3_encode_rne(k)
                    self.v_pool[pid, :, :, :n] = oracle.e4m3_encode_rne(v).transpose(0, 2, 1)
                else:
                    self.k_pool[pid, :, :n] = bits(k)
                    self.v_pool[pid, :, :, :n] = bits(v).transpose(0, 2, 1)

    def at(self, b, t):
        """(page id, slot) of token t of sequence b."""
        for r in self.routes[self.seq_route_begin[b]:self.seq_route_begin[b + 1]]:
            if r[2] <= t < r[3]:
                return int(self.page_ids[r[4] + (t - r[2]) // PAGE]), int((t - r[2]) % PAGE)
        raise IndexError((b, t))

    def device(self, head_major=False):
        """Device tensors of the cache (kf.Shape included, for `Hq` heads given later)."""
        import torch
        from paper_2606_29207_amd.step import _to_dev
        turn = (lambda x: np.ascontiguousarray(np.swapaxes(x, 0, 1))) if head_major else (lambda x: x)
        d = {"k_pool": _to_dev(turn(self.k_pool), "cuda"), "v_pool": _to_dev(turn(self.v_pool), "cuda"),
             "routes": _to_dev(self.routes, "cuda"), "page_ids": _to_dev(self.page_ids, "cuda"),
             "seq_route_begin": _to_dev(self.seq_route_begin, "cuda"),
             "k_scale": None if not self.fp8 else _to_dev(self.k_scale, "cuda"),
             "v_scale": None if not self.fp8 else _to_dev(self.v_scale, "cuda"),
             "err": torch.zeros(1, dtype=torch.int32, device="cuda")}
        return d

    def shape(self, Hq, scale=SCALE, head_major=False):
        from paper_2606_29207_amd import kf
        return kf.make_shape(len(self.lens), Hq, self.H,
                             kf.KV_FP8_E4M3 if self.fp8 else kf.KV_BF16, self.k_pool.shape[0],
                             len(self.page_ids), scale,
                             kf.KV_HEAD_MAJOR if head_major else kf.KV_PAGE_MAJOR)


class Rows:
    """Query rows of the sequences of a cache (counts[b] of sequence b), and for
    trees their drafted K/V and ancestor masks."""

    def __init__(self, cache, counts, G, *, first_pos=None, tree=False, seed=1):
        rng = np.random.default_rng(seed)
        self.cache, self.G, self.counts = cache, G, list(counts)
        self.row_begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        N, H = int(self.row_begin[-1]), cache.H
        self.q = bits(rng.standard_normal((N, H * G, DIM)))
        self.first_pos = self.tree_mask = self.k_draft = self.v_draft = None
        if tree:
            self.k_draft, self.v_draft = (bits(rng.standard_normal((N, H, DIM))) for _ in range(2))
            self.tree_mask = np.array([m & (2 ** 64 - 1) for n in counts for m in tree_masks(n, rng)],
                                      np.uint64).view(np.int64)
        else:
            # by default the rows are their sequence's last tokens
            self.first_pos = np.array(
                [cache.routes[cache.seq_route_begin[b + 1] - 1][3] - n
                 for b, n in enumerate(counts)] if first_pos is None else first_pos, np.int32)

    def oracle(self, scale=SCALE):
        c = self.cache
        return oracle.rows_attn(self.q, self.row_begin, c.k_pool, c.v_pool, c.routes, c.page_ids,
                                c.seq_route_begin, num_kv_heads=c.H, scale=scale,
                                max_pages_per_route=c.max_pages, first_pos=self.first_pos,
                                tree_mask=self.tree_mask, k_draft=self.k_draft,
                                v_draft=self.v_draft, k_scale=c.k_scale, v_scale=c.v_scale)

    def gpu(self, scale=SCALE, head_major=False, stream=None, d=None, pad=0, run=True):
        """The operator's outputs (numpy, float64) and flags; pad: q and the drafted
        rows are parts of wider rows."""
        import torch
        from paper_2606_29207_amd import kf
        from paper_2606_29207_amd.step import _to_dev
        c = self.cache
        d = c.device(head_major) if d is None else d

        def wide(x):
            t = _to_dev(x, "cuda")
            if pad:
                w = torch.full((t.shape[0], t.shape[1] * DIM + pad), float("nan"),
                               dtype=torch.bfloat16, device="cuda")
                w[:, :t.shape[1] * DIM] = t.reshape(t.shape[0], -1)
                t = w[:, :t.shape[1] * DIM].unflatten(1, (t.shape[1], DIM))
            return t

        q = wide(self.q)
        N, Hq = q.shape[:2]
        shape = c.shape(Hq, scale, head_major)
        out = torch.full((N, Hq, DIM), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((N, Hq), float("nan"), device="cuda")
        ws = kf.alloc_rows_workspace(shape, N)
        ws.fill_(0xFF)
        tail = (d["k_pool"], d["v_pool"], d["routes"], c.max_pages, d["page_ids"],
                d["seq_route_begin"], _to_dev(self.row_begin, "cuda"), out, lse, ws, d["err"])
        scales = {"k_scale": d["k_scale"], "v_scale": d["v_scale"]}
        if self.tree_mask is None:
            call = kf.bind_prompt_attn(shape, q, _to_dev(self.first_pos, "cuda"), *tail, **scales)
        else:
            call = kf.bind_tree_attn(shape, q, wide(self.k_draft), wide(self.v_draft),
                                     _to_dev(self.tree_mask, "cuda"), *tail, **scales)
        if not run:
            return call, out, lse, d["err"]
        if stream is not None:
            torch.cuda.synchronize()
        call(stream)
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy(), int(d["err"].item())


def tree_masks(n, rng):
    """Ancestor masks (with the row itself) of n drafted tokens of a random forest."""
    masks = []
    for i in range(n):
        parent = int(rng.integers(-1, i)) if i else -1
        masks.append((1 << i) | (masks[parent] if parent >= 0 else 0))
    return masks


def assert_rows(got, ref, what=""):
    """Outputs against the oracle's.  Two roundings to bf16 at most, each off by
    2^-8 of its value at most: every weight (the weighted |v| then bounds the
    sum's error) and the output; 32-bit sums add far less (2^-16 of the weighted
    |v| is allowed).  lse: the 128 products of a score, added in 32 bits, are off
    by at most 128 x 2^-24 of the sum of their sizes, below 1e-4 for N(0, 1)."""
    out, lse, flags = got
    r_out, r_lse, r_flags, spread = ref
    assert flags == r_flags, f"{what}: flags {flags} != {r_flags}"
    assert np.array_equal(np.isnan(out), np.isnan(r_out)), f"{what}: NaN positions of out differ"
    assert np.array_equal(np.isnan(lse), np.isnan(r_lse)), f"{what}: NaN positions of lse differ"
    assert np.array_equal(np.isneginf(lse), np.isneginf(r_lse)), f"{what}: -inf positions differ"
    fine = ~np.isnan(r_out)
    bound = 2.0 ** -8 * np.abs(r_out) + (2.0 ** -8 + 2.0 ** -16) * spread + 1e-30
    over = np.abs(out - r_out)[fine] - bound[fine]
    assert over.size == 0 or over.max() <= 0, f"{what}: out beyond its bound by {over.max():.3e}"
    fine = np.isfinite(r_lse)
    err = np.abs(lse[fine] - r_lse[fine])
    assert err.size == 0 or err.max() <= 1e-4, f"{what}: lse off by {err.max():.3e}"
