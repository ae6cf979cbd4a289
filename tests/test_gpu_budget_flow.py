"""The operators of a budget as a serving loop uses them: weights from prompts and
decode steps, evictions back and forth between two routes, windows over what is left."""
import numpy as np
import pytest

import oracle
from budget_testlib import (Evictable, assert_evicted, assert_weights, evict_gpu, weights_gpu,
                            window_gpu)
from kf_testlib import assert_close_lse, assert_close_o
from rows_testlib import SCALE, Cache, Rows, assert_rows, bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_prompt_weights_evict_decode_evict_window(gpu, fp8, head_major):
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import DecodeState, _to_dev
    H, G, B = 2, 4, 3
    prompts = [150, 33, 70]
    # two routes a sequence: one that takes the prompt, an empty one
    c = Evictable([0] * B, [0] * B, H=H, fp8=fp8, spare=14, room=[14] * B, seed=1)
    c.max_pages = 14
    c.weights[:] = 0.0
    rng = np.random.default_rng(2)
    q0 = bits(rng.standard_normal((B, H * G, 128)))
    tails = c.seq_route_begin[:-1].astype(np.int32)
    st = DecodeState(q=q0, k_pool=c.k_pool, v_pool=c.v_pool, routes=c.routes, page_ids=c.page_ids,
                     seq_route_begin=c.seq_route_begin, tail_route=tails, scale=SCALE,
                     max_pages_per_route=c.max_pages, k_scale=c.k_scale, v_scale=c.v_scale,
                     kv_layout=kf.KV_HEAD_MAJOR if head_major else None)

    def dev(x):
        return _to_dev(np.asarray(x), "cuda")

    def host(t):
        t = t.contiguous().cpu()
        return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.numpy()

    def pools():
        torch.cuda.synchronize()
        turn = (lambda t: t.transpose(0, 1)) if head_major else (lambda t: t)
        return (host(turn(st.k_pool)), host(turn(st.v_pool)), host(st.weights), host(st.routes),
                host(st.k_scale) if fp8 else None, host(st.v_scale) if fp8 else None, st.flags())

    def held(b):
        return sum(int(r[3] - r[2]) for r in c.routes[c.seq_route_begin[b]:c.seq_route_begin[b + 1]])

    def weigh(r, out_lse, decay, what):
        before = c.weights
        st.attn_weights(dev(r.q), out_lse, dev(r.first_pos), dev(r.row_begin), decay)
        torch.cuda.synchronize()
        lse = out_lse.cpu().numpy()
        ref = oracle.attn_weights(r.q, lse, r.row_begin, r.first_pos, c.k_pool, c.routes, c.page_ids,
                                  before, num_kv_heads=H, scale=SCALE, decay=decay,
                                  max_pages_per_route=c.max_pages, k_scale=c.k_scale)
        got = host(st.weights)
        assert_weights((got, st.flags()), ref, before, what)
        c.weights = got.copy()           # (the next choice follows from these very bits)

    def evict(into, keep, what):
        c.into, c.keep = np.array(into, np.int32), np.array(keep, np.int32)
        ref = oracle.kv_evict(c.k_pool, c.v_pool, c.weights, c.routes, c.page_ids,
                              c.seq_route_begin, c.into, c.keep, max_keep=100, keep_first=2,
                              keep_last=16, max_pages_per_route=c.max_pages, k_scale=c.k_scale,
                              v_scale=c.v_scale)
        st.evict(dev(c.into), dev(c.keep), 100, 2, 16)
        st.tail_route.copy_(dev(c.into))
        assert_evicted(pools(), ref, what)
        c.k_pool, c.v_pool, c.weights, c.routes, c.k_scale, c.v_scale = ref[:6]

    def decode(tail, what):
        kn, vn = (bits(rng.standard_normal((B, H, 128))) for _ in range(2))
        st.step_fused(dev(kn), dev(vn))
        got = oracle.kv_append(c.k_pool, c.v_pool, c.routes, c.page_ids, tail, kn, vn,
                               *((c.k_scale, c.v_scale) if fp8 else ()))
        c.k_pool, c.v_pool, c.routes = got[0], got[1], got[-2]
        if fp8:
            c.k_scale, c.v_scale = got[2], got[3]
        o, l, _ = oracle.partial_attn(q0, c.k_pool, c.v_pool, c.routes, c.page_ids, num_kv_heads=H,
                                      scale=SCALE, max_pages_per_route=c.max_pages,
                                      k_scale=c.k_scale, v_scale=c.v_scale)
        out, lse, _ = oracle.merge_partials(o, l, c.seq_route_begin)
        torch.cuda.synchronize()
        assert_close_o(st.out.double().cpu().numpy(), out, what)
        assert_close_lse(st.lse.double().cpu().numpy(), lse, what)
        # the step's weights: one row a sequence, at its newest token
        r = Rows(c, [1] * B, G, first_pos=[int(c.routes[t][3]) - 1 for t in tail])
        r.q = q0
        weigh(r, st.lse, 0.9, what)

    # the prompts
    k, v = (bits(rng.standard_normal((sum(prompts), H, 128))) for _ in range(2))
    counts = np.zeros(len(c.routes), int)
    counts[tails] = prompts
    begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    st.append_rows(dev(k), dev(v), dev(begin))
    got = oracle.kv_append_rows(c.k_pool, c.v_pool, c.routes, c.page_ids, k, v, begin, None,
                                num_seqs=B, k_scale=c.k_scale, v_scale=c.v_scale)
    c.k_pool, c.v_pool, c.routes = got[0], got[1], got[-2]
    if fp8:
        c.k_scale, c.v_scale = got[2], got[3]
    r = Rows(c, prompts, G, first_pos=[0] * B, seed=5)
    out, lse = st.prompt_attn(dev(r.q), dev(r.first_pos), dev(r.row_begin))
    torch.cuda.synchronize()
    weigh(r, lse, 1.0, "prompt")
    total = [c.weights[c.page_ids[c.routes[t][4] + np.arange(prompts[b]) // 16], :,
                       np.arange(prompts[b]) % 16].sum(0) for b, t in enumerate(tails)]
    for b in range(B):                   # every row gives each of its heads a weight of one
        assert np.allclose(total[b], prompts[b] * G, rtol=1e-3)
    # down to a budget, decode steps, and back to it between the same two routes
    other = c.seq_route_begin[1:].astype(np.int32) - 1
    evict(other, [60, 40, 16], "first eviction")
    assert [held(b) for b in range(B)] == [60, 33, 16]
    for i in range(3):
        decode(other, f"decode {i}")
    evict(tails, [30, 34, 16], "second eviction")
    assert [held(b) for b in range(B)] == [30, 34, 16]
    for i in range(2):
        decode(tails, f"decode {3 + i}")
    # windows over what is left
    last = [int(c.routes[t][3]) - 1 for t in tails]
    for sinks, window in ((0, 8), (4, 12), (0, 1000)):
        r = Rows(c, [1] * B, G, first_pos=last, seed=9)
        out, lse = st.window_attn(dev(r.q), dev(r.first_pos), dev(r.row_begin), sinks, window)
        torch.cuda.synchronize()
        ref = oracle.rows_attn(r.q, r.row_begin, c.k_pool, c.v_pool, c.routes, c.page_ids,
                               c.seq_route_begin, num_kv_heads=H, scale=SCALE,
                               max_pages_per_route=c.max_pages, first_pos=r.first_pos,
                               k_scale=c.k_scale, v_scale=c.v_scale, sinks=sinks, window=window)
        assert_rows((out.double().cpu().numpy(), lse.double().cpu().numpy(), st.flags()), ref)


def test_a_graph_of_weights_and_eviction_after_decode_steps(gpu):
    """One captured graph: decode step, its weights, eviction; replayed from the same
    state, with other work between, it leaves the same bits every time."""
    import torch
    from paper_2606_29207_amd.step import DecodeState, _to_dev
    H, G, B = 2, 4, 2
    c = Evictable([90, 40], [48, 32], H=H, spare=4, room=[3, 2], seed=4)
    rng = np.random.default_rng(2)
    q0 = bits(rng.standard_normal((B, H * G, 128)))
    tails = (c.into - 1).astype(np.int32)
    st = DecodeState(q=q0, k_pool=c.k_pool, v_pool=c.v_pool, routes=c.routes, page_ids=c.page_ids,
                     seq_route_begin=c.seq_route_begin, tail_route=tails, scale=SCALE,
                     max_pages_per_route=c.max_pages)
    st.weights.copy_(torch.from_numpy(c.weights))
    kn, vn = (_to_dev(bits(rng.standard_normal((B, H, 128))), "cuda") for _ in range(2))
    pos = _to_dev(np.array([90, 40], np.int32), "cuda")
    rows = _to_dev(np.arange(B + 1, dtype=np.int32), "cuda")
    into, keep = _to_dev(c.into.astype(np.int32), "cuda"), _to_dev(c.keep, "cuda")
    state = [st.k_pool, st.v_pool, st.weights, st.routes]
    start = [t.clone() for t in state]

    def loop():
        st.step_fused(kn, vn)
        st.attn_weights(st.q, st.lse, pos, rows)
        st.evict(into, keep, 48, 2, 8)

    loop()
    torch.cuda.synchronize()
    want = [t.clone() for t in state]
    assert st.flags() == 0
    assert (want[3][into.long(), 3] - want[3][into.long(), 2]).tolist() == [48, 32]
    for t, s in zip(state, start):
        t.copy_(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loop()
    for i in range(4):
        for t, s in zip(state, start):
            t.copy_(s)
        (torch.ones(1 << 16, device="cuda") * i).sum().item()
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip(state, want):
            assert torch.equal(t.view(torch.uint8), w.view(torch.uint8)), i


def test_weights_are_not_first_used_in_a_capture(gpu):
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import DecodeState
    c = Cache([40], H=1, seed=1)
    st = DecodeState(q=bits(np.zeros((1, 4, 128))), k_pool=c.k_pool, v_pool=c.v_pool,
                     routes=c.routes, page_ids=c.page_ids, seq_route_begin=c.seq_route_begin,
                     tail_route=np.zeros(1, np.int32), scale=SCALE, max_pages_per_route=c.max_pages)
    x = torch.zeros(4, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        with pytest.raises(kf.KFError, match="before a capture"):
            st.weights
        x += 1                           # (a graph of something)
    g.replay()
    assert (st.weights == 0).all() and st.weights is st.weights


def test_calls_on_streams_at_once(gpu):
    """A window, weights and an eviction over caches of their own, in flight together."""
    import torch
    c1, c2 = Cache([3000, 900], H=2, part=1024, seed=1), Cache([2500, 400, 70], H=2, fp8=True, seed=2)
    c3 = Evictable([90000, 2000], [3000, 500], H=2, part=9000, seed=3)
    r1, r2 = Rows(c1, [300, 20], 4, seed=3), Rows(c2, [30, 400, 3], 4, seed=4)
    lse = r2.oracle()[1].astype(np.float32)
    w0 = np.zeros((c2.k_pool.shape[0], 2, 16), np.float32)
    alone = window_gpu(r1, 4, 500), weights_gpu(r2, lse, w0, 0.0), evict_gpu(c3, 4, 100)
    call1, out, l1, e1 = window_gpu(r1, 4, 500, run=False)
    call2, w, e2 = weights_gpu(r2, lse, w0, 0.0, run=False)
    call3, w3, d3 = evict_gpu(c3, 4, 100, run=False)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    routes = d3["routes"].clone()
    for _ in range(4):
        for call, s in zip((call1, call2, call3), streams):
            call(s)
        with torch.cuda.stream(streams[2]):
            done = d3["routes"].clone()
            d3["routes"].copy_(routes)
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), alone[0][0])
    assert np.array_equal(w.cpu().numpy(), alone[1][0])
    assert np.array_equal(done.cpu().numpy(), alone[2][3])
    assert np.array_equal(w3.cpu().numpy(), alone[2][2])
    assert int(e1.item()) == int(e2.item()) == int(d3["err"].item()) == 0


def test_pools_beyond_32_bit_offsets(gpu):
    """Pages and weights behind 4 GiB: a small cache in the last pages of large pools."""
    import torch
    from paper_2606_29207_amd import kf
    H, G, P = 8, 4, 140000               # 4.6 GB a pool
    c = Cache([300], H=H, seed=3)
    n = c.k_pool.shape[0]
    r = Rows(c, [100], G, seed=3)
    lse = r.oracle()[1].astype(np.float32)
    w0 = np.zeros((n, H, 16), np.float32)
    want = window_gpu(r, 4, 50), weights_gpu(r, lse, w0, 0.0)
    d = c.device()
    big = {}
    for k in ("k_pool", "v_pool"):
        big[k] = torch.zeros((P,) + tuple(d[k].shape[1:]), dtype=torch.bfloat16, device="cuda")
        big[k][P - n:] = d[k]
    d.update(big)
    d["page_ids"] = d["page_ids"] + (P - n)
    shape = kf.make_shape(1, H * G, H, kf.KV_BF16, P, d["page_ids"].numel(), SCALE)
    from paper_2606_29207_amd.step import _to_dev
    q, pos, begin = (_to_dev(x, "cuda") for x in (r.q, r.first_pos, r.row_begin))
    out = torch.empty((100, H * G, 128), dtype=torch.bfloat16, device="cuda")
    l = torch.empty((100, H * G), device="cuda")
    kf.window_attn(shape, q, pos, 4, 50, d["k_pool"], d["v_pool"], d["routes"], c.max_pages,
                   d["page_ids"], d["seq_route_begin"], begin, out, l,
                   kf.alloc_rows_workspace(shape, 100), d["err"])
    w = torch.zeros((P, H, 16), device="cuda")
    kf.attn_weights(shape, q, _to_dev(lse, "cuda"), pos, d["k_pool"], d["routes"], c.max_pages,
                    d["page_ids"], begin, 0.0, w, d["err"])
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want[0][0])
    assert np.array_equal(w[P - n:].cpu().numpy(), want[1][0]) and int(d["err"].item()) == 0
    # the tokens move to the first pages
    rows = torch.cat((d["routes"], torch.tensor([[0, 1, 0, 0, d["page_ids"].numel(), 5]],
                                                dtype=torch.int32, device="cuda")))
    ids = torch.cat((d["page_ids"], torch.arange(5, dtype=torch.int32, device="cuda")))
    shape = kf.make_shape(1, H * G, H, kf.KV_BF16, P, ids.numel(), SCALE)
    i32 = dict(dtype=torch.int32, device="cuda")
    kf.kv_evict(shape, d["k_pool"], d["v_pool"], w, rows, 20, ids, torch.tensor([0, 2], **i32),
                torch.tensor([1], **i32), torch.tensor([80], **i32), 80, 80, 0, d["err"])
    torch.cuda.synchronize()
    assert rows[:, 3].tolist() == [0, 80] and int(d["err"].item()) == 0
    src = d["page_ids"][:5].long()
    for t in (d["k_pool"], d["v_pool"], w):
        assert torch.equal(t[:5], t[src])
