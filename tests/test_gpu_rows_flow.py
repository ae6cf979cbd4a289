"""The row operators as a serving loop uses them together, over one state:
prompts are appended and attended in two chunks, a decode step follows, trees are
drafted and attended, their accepted paths appended, and another decode step
reads all of it.  Every stage against the fp64 oracle on the oracle's own copy of
the cache, pools, scales and routes bit for bit."""
import numpy as np
import pytest

import oracle
from kf_testlib import assert_close_lse, assert_close_o
from rows_testlib import SCALE, Cache, Rows, assert_rows, bits

pytestmark = pytest.mark.gpu


def _host(t):
    import torch
    t = t.cpu()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.numpy()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_prompt_decode_tree_accept_decode(gpu, fp8, head_major):
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import DecodeState, _to_dev
    H, G, B = 2, 4, 3
    prompts, chunk = [150, 33, 70], [100, 33, 64]
    # empty caches of one route each, pages reserved for everything that follows
    c = Cache([0] * B, H=H, fp8=fp8, spare=14, seed=1)
    c.max_pages = 14
    rng = np.random.default_rng(2)
    q0 = bits(rng.standard_normal((B, H * G, 128)))
    st = DecodeState(q=q0, k_pool=c.k_pool, v_pool=c.v_pool, routes=c.routes, page_ids=c.page_ids,
                     seq_route_begin=c.seq_route_begin, tail_route=np.arange(B), scale=SCALE,
                     max_pages_per_route=c.max_pages, k_scale=c.k_scale, v_scale=c.v_scale,
                     kv_layout=kf.KV_HEAD_MAJOR if head_major else None)

    def dev(x, dtype=None):
        return _to_dev(np.asarray(x) if dtype is None else np.asarray(x, dtype), "cuda")

    def same_cache(what):
        torch.cuda.synchronize()
        assert st.flags() == 0, what
        names = ["k_pool", "v_pool"] + (["k_scale", "v_scale"] if fp8 else [])
        for n in names:
            t = _host(getattr(st, n))
            if head_major and n.endswith("pool"):
                t = np.swapaxes(t, 0, 1)
            a, b = np.ascontiguousarray(t), getattr(c, n)
            assert np.array_equal(a.view(np.uint8), np.ascontiguousarray(b).view(np.uint8)), (what, n)
        assert np.array_equal(_host(st.routes), c.routes), what

    def append(k, v, counts, row_list=None):
        begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        st.append_rows(dev(k), dev(v), dev(begin),
                       None if row_list is None else dev(row_list, np.int32))
        got = oracle.kv_append_rows(c.k_pool, c.v_pool, c.routes, c.page_ids, k, v, begin, row_list,
                                    num_seqs=B, k_scale=c.k_scale, v_scale=c.v_scale)
        c.k_pool, c.v_pool, c.routes = got[0], got[1], got[-2]
        if fp8:
            c.k_scale, c.v_scale = got[2], got[3]
        assert got[-1] == 0

    def rows(n):
        return tuple(bits(rng.standard_normal((n, H, 128))) for _ in range(2))

    def decode(what):
        kn, vn = rows(B)
        st.step_fused(dev(kn), dev(vn))
        got = oracle.kv_append(c.k_pool, c.v_pool, c.routes, c.page_ids, np.arange(B), kn, vn,
                               *((c.k_scale, c.v_scale) if fp8 else ()))
        c.k_pool, c.v_pool, c.routes = got[0], got[1], got[-2]
        if fp8:
            c.k_scale, c.v_scale = got[2], got[3]
        same_cache(what)
        o, l, _ = oracle.partial_attn(q0, c.k_pool, c.v_pool, c.routes, c.page_ids, num_kv_heads=H,
                                      scale=SCALE, max_pages_per_route=c.max_pages,
                                      k_scale=c.k_scale, v_scale=c.v_scale)
        out, lse, _ = oracle.merge_partials(o, l, c.seq_route_begin)
        assert_close_o(st.out.double().cpu().numpy(), out, what)
        assert_close_lse(st.lse.double().cpu().numpy(), lse, what)

    # the prompts in two chunks
    done = [0] * B
    for take in (chunk, [n - m for n, m in zip(prompts, chunk)]):
        append(*rows(sum(take)), take)
        same_cache("prompt")
        r = Rows(c, take, G, first_pos=done, seed=sum(take))
        out, lse = st.prompt_attn(dev(r.q), dev(r.first_pos), dev(r.row_begin))
        torch.cuda.synchronize()
        assert_rows((out.double().cpu().numpy(), lse.double().cpu().numpy(), st.flags()), r.oracle())
        done = [a + b for a, b in zip(done, take)]
    decode("first decode step")
    # drafted trees; the accepted rows are each tree's path to its last leaf
    counts = [12, 1, 7]
    r = Rows(c, counts, G, tree=True, seed=9)
    out, lse = st.tree_attn(dev(r.q), dev(r.k_draft), dev(r.v_draft), dev(r.tree_mask),
                            dev(r.row_begin))
    torch.cuda.synchronize()
    assert_rows((out.double().cpu().numpy(), lse.double().cpu().numpy(), st.flags()), r.oracle())
    path = [[int(r.row_begin[b]) + j for j in range(n) if int(r.tree_mask[r.row_begin[b + 1] - 1]) >> j & 1]
            for b, n in enumerate(counts)]
    append(r.k_draft, r.v_draft, [len(p) for p in path], sum(path, []))
    same_cache("accepted rows")
    decode("second decode step")


def test_calls_on_two_streams_at_once(gpu):
    """Prompts and trees of two caches, each with its own workspace, in flight
    together; the same bits as one after another."""
    import torch
    c1, c2 = Cache([3000, 900], H=2, part=1024, seed=1), Cache([2500, 40, 7], H=2, fp8=True, seed=2)
    r1, r2 = Rows(c1, [300, 20], 4, seed=3), Rows(c2, [30, 12, 3], 4, tree=True, seed=4)
    alone = [r.gpu() for r in (r1, r2)]
    calls = [r.gpu(run=False) for r in (r1, r2)]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for (call, *_), s in zip(calls, streams):
            call(s)
    torch.cuda.synchronize()
    for (call, out, lse, err), (o, l, f) in zip(calls, alone):
        assert int(err.item()) == f == 0
        assert np.array_equal(out.double().cpu().numpy(), o)
        assert np.array_equal(lse.double().cpu().numpy(), l)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_pools_beyond_32_bit_offsets(gpu, fp8, head_major):
    """A small cache whose pages lie at the end of pools of more than 4 GiB."""
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import _to_dev
    H, G = 8, 4
    c = Cache([200, 70], H=H, fp8=fp8, seed=3, spare=4)
    P = (5 << 30) // (H * 2048 * (1 if fp8 else 2))
    small = c.device(head_major)
    n = c.k_pool.shape[0]
    big = {}
    for name in ("k_pool", "v_pool"):
        t = small[name]
        shape = (H, P) + tuple(t.shape[2:]) if head_major else (P,) + tuple(t.shape[1:])
        big[name] = torch.zeros(shape, dtype=t.dtype, device="cuda")
        (big[name][:, P - n:] if head_major else big[name][P - n:]).copy_(t)
    if fp8:
        for name in ("k_scale", "v_scale"):
            big[name] = torch.ones((P, H), device="cuda")
            big[name][P - n:].copy_(small[name])
    ids = small["page_ids"] + (P - n)
    shape = kf.make_shape(2, H * G, H, kf.KV_FP8_E4M3 if fp8 else kf.KV_BF16, P, ids.numel(), 0.1,
                          kf.KV_HEAD_MAJOR if head_major else kf.KV_PAGE_MAJOR)
    scales = {k: big.get(k) for k in ("k_scale", "v_scale")}
    err = small["err"]
    # rows appended behind both sequences, then attended
    rng = np.random.default_rng(1)
    k, v = (bits(rng.standard_normal((60, H, 128))) for _ in range(2))
    begin = np.array([0, 40, 60], np.int32)
    kf.kv_append_rows(shape, big["k_pool"], big["v_pool"], _to_dev(k, "cuda"), _to_dev(v, "cuda"),
                      small["routes"], _to_dev(begin, "cuda"), ids, err, **scales)
    got = oracle.kv_append_rows(c.k_pool, c.v_pool, c.routes, c.page_ids, k, v, begin, num_seqs=2,
                                k_scale=c.k_scale, v_scale=c.v_scale)
    c.k_pool, c.v_pool, c.routes = got[0], got[1], got[-2]
    if fp8:
        c.k_scale, c.v_scale = got[2], got[3]
    for tree in (False, True):
        r = Rows(c, [40, 20], G, tree=tree, seed=5)
        q = _to_dev(r.q, "cuda")
        out = torch.empty((60, H * G, 128), dtype=torch.bfloat16, device="cuda")
        lse = torch.empty((60, H * G), device="cuda")
        tail = (big["k_pool"], big["v_pool"], small["routes"], c.max_pages, ids,
                small["seq_route_begin"], _to_dev(r.row_begin, "cuda"), out, lse,
                kf.alloc_rows_workspace(shape, 60), err)
        if tree:
            kf.tree_attn(shape, q, _to_dev(r.k_draft, "cuda"), _to_dev(r.v_draft, "cuda"),
                         _to_dev(r.tree_mask, "cuda"), *tail, **scales)
        else:
            kf.prompt_attn(shape, q, _to_dev(r.first_pos, "cuda"), *tail, **scales)
        torch.cuda.synchronize()
        ref = r.oracle(0.1)
        assert_rows((out.double().cpu().numpy(), lse.double().cpu().numpy(), int(err.item())), ref)
    for name in ("k_pool", "v_pool"):
        t = big[name][:, P - n:].transpose(0, 1) if head_major else big[name][P - n:]
        assert np.array_equal(_host(t.contiguous()), getattr(c, name)), name
    del big
    torch.cuda.empty_cache()
