"""Pins of the oracle's window attention, attention weights and eviction, each against
something other than the oracle itself (no GPU)."""
import numpy as np
import pytest
import torch

import oracle
from budget_testlib import Evictable, evict_oracle, start_weights, window_oracle
from rows_testlib import SCALE, Cache, Rows


def _tokens(c, b, pool, scale, is_v):
    """K or V [n, H, 128] of sequence b, token by token from the tables."""
    out = []
    for r in c.routes[c.seq_route_begin[b]:c.seq_route_begin[b + 1]]:
        for j in range(int(r[3]) - int(r[2])):
            pid = int(c.page_ids[r[4] + j // 16])
            x = pool[pid, :, :, j % 16] if is_v else pool[pid, :, j % 16]
            if c.fp8:
                x = torch.from_numpy(x.copy()).view(torch.float8_e4m3fn).double().numpy() * \
                    scale[pid][:, None]
            else:
                x = torch.from_numpy(x.view(np.int16).copy()).view(torch.bfloat16).double().numpy()
            out.append(x)
    return torch.from_numpy(np.array(out).reshape(-1, c.H, 128))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("sinks,window", [(0, 5), (3, 8), (10, 0), (0, 100)])
def test_windows_against_sdpa(fp8, sinks, window):
    lens, counts, G = [40, 7, 25], [10, 7, 3], 3
    c = Cache(lens, H=2, fp8=fp8, part=16, seed=1)
    r = Rows(c, counts, G, seed=2)
    out, lse, flags, _ = window_oracle(r, sinks, window)
    assert flags == 0
    for b, n in enumerate(counts):
        k = _tokens(c, b, c.k_pool, c.k_scale, False).transpose(0, 1)
        v = _tokens(c, b, c.v_pool, c.v_scale, True).transpose(0, 1)
        q = torch.from_numpy(oracle.bf16_to_f64(r.q[r.row_begin[b]:r.row_begin[b + 1]])).transpose(0, 1)
        p = torch.arange(lens[b] - n, lens[b])[:, None]
        t = torch.arange(lens[b])[None]
        band = (t <= p) & ((p - t < window) | (t < sinks))
        got = torch.from_numpy(out[r.row_begin[b]:r.row_begin[b + 1]]).transpose(0, 1)
        seen = band.any(1)
        ref = torch.nn.functional.scaled_dot_product_attention(
            q[:, seen], k, v, attn_mask=band[seen], scale=SCALE, enable_gqa=True)
        assert torch.allclose(got[:, seen], ref, atol=1e-12)
        assert (got[:, ~seen] == 0).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("decay", [0.0, 0.75])
def test_weights_against_a_softmax(fp8, decay):
    lens, counts, G = [40, 7, 25], [10, 7, 3], 3
    c = Cache(lens, H=2, fp8=fp8, part=16, seed=1)
    r = Rows(c, counts, G, seed=2)
    w0 = start_weights(c)
    lse = r.oracle()[1]
    got, flags, terms = oracle.attn_weights(r.q, lse, r.row_begin, r.first_pos, c.k_pool, c.routes,
                                            c.page_ids, w0, num_kv_heads=2, scale=SCALE, decay=decay,
                                            max_pages_per_route=c.max_pages, k_scale=c.k_scale)
    assert flags == 0 and terms == 30
    touched = np.zeros_like(w0, bool)
    for b, n in enumerate(counts):
        k = _tokens(c, b, c.k_pool, c.k_scale, False).transpose(0, 1)          # [H, t, 128]
        q = torch.from_numpy(oracle.bf16_to_f64(r.q[r.row_begin[b]:r.row_begin[b + 1]]))
        s = torch.einsum("ihgd,htd->ihgt", q.view(n, 2, G, 128), k) * SCALE
        future = torch.arange(lens[b])[None] > torch.arange(lens[b] - n, lens[b])[:, None]
        p = torch.softmax(s.masked_fill(future[:, None, None], -torch.inf), -1).sum((0, 2))
        for t in range(lens[b]):
            pid, slot = c.at(b, t)
            touched[pid, :, slot] = True
            old = decay * w0[pid, :, slot].astype(np.float64) if t < lens[b] - n else 0.0
            assert np.allclose(got[pid, :, slot], old + p[:, t].numpy(), atol=1e-12)
    assert np.array_equal(got[~touched], w0[~touched].astype(np.float64))


@pytest.mark.parametrize("fp8", [False, True])
def test_evictions_against_a_sort(fp8):
    lens, keep, first, last = [100, 37, 20], [41, 16, 50], 3, 9
    c = Evictable(lens, keep, H=2, fp8=fp8, part=40, seed=1)
    before = [x if x is None else x.copy() for x in (c.k_pool, c.v_pool, c.weights, c.k_scale, c.v_scale)]
    k, v, w, routes, ks, vs, flags = evict_oracle(c, first, last)
    assert flags == 0
    for b, L in enumerate(lens):
        to = int(c.into[b])
        K = min(L, keep[b])
        rows = routes[c.seq_route_begin[b]:c.seq_route_begin[b + 1]]
        assert (rows[:-1, 3] == rows[:-1, 2]).all() and rows[-1, 3] - rows[-1, 2] == K
        place = [c.at(b, t) for t in range(L)]
        for g in range(2):
            weight = [float(c.weights[p, g, s]) for p, s in place]
            mid = sorted(range(first, L - last), key=lambda t: (-weight[t], t)) if K < L else range(L)
            stay = sorted(set(range(min(first, L))) | set(range(max(0, L - last), L)) |
                          set(list(mid)[:K - first - last] if K < L else mid))
            assert len(stay) == K
            for i, t in enumerate(stay):
                sp, ss = place[t]
                dp, ds = int(c.page_ids[c.routes[to][4] + i // 16]), i % 16
                assert w[dp, g, ds] == before[2][sp, g, ss]
                if not fp8:
                    assert np.array_equal(k[dp, g, ds], before[0][sp, g, ss])
                    assert np.array_equal(v[dp, g, :, ds], before[1][sp, g, :, ss])
                    continue
                for new, sc, old, was, is_v in ((k, ks, before[0], before[3], False),
                                                (v, vs, before[1], before[4], True)):
                    x = (old[sp, g, :, ss] if is_v else old[sp, g, ss]).copy()
                    y = (new[dp, g, :, ds] if is_v else new[dp, g, ds]).copy()
                    group = stay[i // 16 * 16:i // 16 * 16 + 16]
                    assert sc[dp, g] == max(was[place[u][0], g] for u in group)
                    value = torch.from_numpy(x).view(torch.float8_e4m3fn).float() * was[sp, g] / sc[dp, g]
                    assert np.array_equal(value.to(torch.float8_e4m3fn).view(torch.uint8).numpy(), y)


def test_ties_and_nan_of_an_eviction():
    c = Evictable([6], [3], H=1, seed=1)
    pid = int(c.page_ids[0])
    c.weights[pid, 0, :6] = [np.nan, 1.0, 0.0, 1.0, -0.0, 1.0]
    k, _, _, _, _, _, flags = evict_oracle(c, 0, 0)
    to = int(c.page_ids[c.routes[c.into[0]][4]])
    assert flags == 0 and np.array_equal(k[to, 0, :3], c.k_pool[pid, 0, [1, 3, 5]])
    c.keep[:] = 5
    k = evict_oracle(c, 0, 0)[0]
    assert np.array_equal(k[to, 0, :5], c.k_pool[pid, 0, 1:6])       # NaN goes first
    c.keep[:] = 4
    k = evict_oracle(c, 0, 0)[0]
    assert np.array_equal(k[to, 0, :4], c.k_pool[pid, 0, [1, 2, 3, 5]])  # 0 equals -0: the earlier
