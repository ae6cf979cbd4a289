"""Pins of the oracle's row operators, each against something other than the
oracle itself (no GPU)."""
import numpy as np
import pytest
import torch

import oracle
from rows_testlib import DIM, SCALE, Cache, Rows, bits, tree_masks


def _gathered(c, b, H):
    """K, V [H, n, 128] of sequence b, token by token from the tables."""
    ks, vs = [], []
    for r in c.routes[c.seq_route_begin[b]:c.seq_route_begin[b + 1]]:
        for j in range(r[3] - r[2]):
            pid, slot = int(c.page_ids[r[4] + j // 16]), j % 16
            k, v = c.k_pool[pid, :, slot], c.v_pool[pid, :, :, slot]
            if c.fp8:
                k, v = (torch.from_numpy(x.copy()).view(torch.float8_e4m3fn).double().numpy() * s[pid][:, None]
                        for x, s in ((k, c.k_scale), (v, c.v_scale)))
            else:
                k, v = (torch.from_numpy(x.view(np.int16).copy()).view(torch.bfloat16).double().numpy()
                        for x in (k, v))
            ks.append(k)
            vs.append(v)
    none = np.zeros((0, H, DIM))
    return (np.concatenate([none, np.array(ks).reshape(-1, H, DIM)]).transpose(1, 0, 2),
            np.concatenate([none, np.array(vs).reshape(-1, H, DIM)]).transpose(1, 0, 2))


def _sdpa(q, k, v, mask, scale):
    out = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q), torch.from_numpy(k), torch.from_numpy(v),
        attn_mask=torch.from_numpy(mask), scale=scale, enable_gqa=True)
    return out.numpy()


@pytest.mark.parametrize("fp8", [False, True])
def test_prompts_against_sdpa(fp8):
    lens = [40, 7, 25]
    c = Cache(lens, H=2, fp8=fp8, part=16, seed=1)
    r = Rows(c, [10, 7, 3], 3, seed=2)
    out, lse, flags, spread = r.oracle()
    assert flags == 0
    for b, n in enumerate([10, 7, 3]):
        k, v = _gathered(c, b, 2)
        rows = slice(r.row_begin[b], r.row_begin[b + 1])
        q = oracle.bf16_to_f64(r.q[rows]).transpose(1, 0, 2)
        mask = np.arange(lens[b])[None, :] <= (lens[b] - n + np.arange(n))[:, None]
        assert np.allclose(out[rows].transpose(1, 0, 2), _sdpa(q, k, v, mask, SCALE), atol=1e-12)
        assert np.allclose(spread[rows].transpose(1, 0, 2), _sdpa(q, k, np.abs(v), mask, SCALE),
                           atol=1e-12)
        s = np.where(mask, np.einsum("hid,htd->hit", q, np.repeat(k, 3, 0)) * SCALE, -np.inf)
        assert np.allclose(lse[rows].T, torch.logsumexp(torch.from_numpy(s), -1).numpy(), atol=1e-12)


def test_trees_against_sdpa():
    lens, counts = [20, 0, 33], [6, 4, 9]
    c = Cache(lens, H=2, part=16, seed=1)
    r = Rows(c, counts, 2, tree=True, seed=3)
    out, _, flags, _ = r.oracle()
    assert flags == 0
    for b, n in enumerate(counts):
        k, v = _gathered(c, b, 2)
        rows = slice(r.row_begin[b], r.row_begin[b + 1])
        kd, vd = (oracle.bf16_to_f64(x[rows]).transpose(1, 0, 2) for x in (r.k_draft, r.v_draft))
        drafted = np.array([[bool(int(m) >> j & 1) for j in range(n)] for m in r.tree_mask[rows]])
        mask = np.concatenate([np.ones((n, lens[b]), bool), drafted], 1)
        q = oracle.bf16_to_f64(r.q[rows]).transpose(1, 0, 2)
        want = _sdpa(q, np.concatenate([k, kd], 1), np.concatenate([v, vd], 1), mask, SCALE)
        assert np.allclose(out[rows].transpose(1, 0, 2), want, atol=1e-12)


def test_a_chain_of_drafts_is_a_prompt():
    """Drafted tokens of one chain see what the same tokens see in the cache."""
    c = Cache([30], H=2, spare=1, seed=5)
    r = Rows(c, [6], 2, tree=True, seed=6)
    r.tree_mask[:] = [(2 << i) - 1 for i in range(6)]
    tree = r.oracle()
    c.k_pool, c.v_pool, c.routes, f = oracle.kv_append_rows(
        c.k_pool, c.v_pool, c.routes, c.page_ids, r.k_draft, r.v_draft, [0, 6], num_seqs=1)
    p = Rows(c, [6], 2, seed=6)
    p.q = r.q
    prompt = p.oracle()
    assert f == tree[2] == prompt[2] == 0
    assert np.allclose(tree[0], prompt[0], atol=1e-13) and np.allclose(tree[1], prompt[1], atol=1e-13)


def test_rows_that_see_nothing():
    c = Cache([5, 0], H=1, first=[10, 0])
    r = Rows(c, [3, 1], 2, first_pos=[8, 0])
    out, lse, flags, _ = r.oracle()
    assert flags == 0 and np.isneginf(lse[[0, 1, 3]]).all() and not out[[0, 1, 3]].any()
    assert np.isfinite(lse[2]).all()
    # a single visible token is returned as it is
    pid, slot = c.at(0, 10)
    assert np.allclose(out[2], oracle.bf16_to_f64(c.v_pool[pid, 0, :, slot]))


@pytest.mark.parametrize("fp8", [False, True])
def test_append_rows_are_single_appends(fp8):
    rng = np.random.default_rng(4)
    n, B = 19, 2
    c = Cache([7, 30], H=2, fp8=fp8, spare=4, seed=1)
    size = np.exp(rng.uniform(0, 6, (B * n, 2, 1)))
    k, v = (bits(rng.standard_normal((B * n, 2, DIM)) * size) for _ in range(2))
    order = rng.permutation(B * n)
    got = oracle.kv_append_rows(c.k_pool, c.v_pool, c.routes, c.page_ids, k, v, [0, n, 2 * n], order,
                                num_seqs=B, k_scale=c.k_scale, v_scale=c.v_scale)
    state = [c.k_pool, c.v_pool] + ([c.k_scale, c.v_scale] if fp8 else []) + [c.routes]
    for i in range(n):
        pick = [order[i], order[n + i]]
        res = oracle.kv_append(state[0], state[1], state[-1], c.page_ids, np.arange(B), k[pick],
                               v[pick], *state[2:-1])
        state = list(res[:-1])
        assert res[-1] == 0
    assert got[-1] == 0
    for a, b in zip(got[:-1], state):
        assert np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


def test_tree_masks_are_ancestors():
    for n in (1, 5, 64):
        masks = tree_masks(n, np.random.default_rng(n))
        for i, m in enumerate(masks):
            assert m >> i & 1 and m >> (i + 1) == 0
            up = [j for j in range(i) if m >> j & 1]
            if up:  # the parent's own mask is the rest
                assert masks[up[-1]] == m ^ (1 << i)


@pytest.mark.parametrize("mutant", ["later", "draft", "scale", "head"])
def test_planted_mistakes_are_seen(mutant):
    """What the GPU comparison would have to catch, planted in a second oracle call."""
    c = Cache([40], H=2, seed=8)
    r = Rows(c, [12], 2, tree=mutant == "draft", seed=9)
    out, _, _, spread = r.oracle()
    if mutant == "later":
        r.first_pos = r.first_pos + 1
    elif mutant == "draft":
        r.tree_mask[5] ^= 1 << 5
    elif mutant == "head":
        r.q = r.q[:, [0, 2, 1, 3]]
    wrong = r.oracle(SCALE * (1.02 if mutant == "scale" else 1))[0]
    bound = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2.0 ** -16) * spread
    assert (np.abs(wrong - out) > bound).any()
