"""kf_kv_evict against the oracle, bit for bit: pools, scales, weights, routes."""
import numpy as np
import pytest

from budget_testlib import (Evictable, assert_evicted, evict_gpu, evict_oracle, evict_parts,
                            evict_result)

pytestmark = pytest.mark.gpu


def check(c, first, last, what="", **kw):
    ref = evict_oracle(c, first, last, kw.get("max_keep"))
    got = evict_gpu(c, first, last, **kw)
    assert_evicted(got, ref, what)
    return got


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_sequences_of_several_routes(gpu, fp8, head_major):
    c = Evictable([300, 1, 77, 640, 16], [100, 5, 40, 333, 16], H=3, fp8=fp8, part=112, seed=1)
    check(c, 4, 20, head_major=head_major)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("keep", [0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 99, 100, 101, 1000])
def test_every_budget(gpu, keep, fp8):
    c = Evictable([100], [keep], H=2, fp8=fp8, part=40, seed=keep)
    check(c, 2, 7)


@pytest.mark.parametrize("first,last", [(0, 0), (0, 50), (50, 0), (10, 30), (60, 60), (1000, 3),
                                        (0, 1000), (49, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_first_and_last_tokens(gpu, first, last):
    c = Evictable([200, 50, 30], [50, 50, 50], H=2, part=64, seed=2)
    check(c, first, last)


@pytest.mark.parametrize("L", [1, 63, 64, 65, 1023, 1024, 1025, 5000, 34815, 34816, 34817, 50000])
def test_lengths(gpu, L):
    c = Evictable([L], [max(1, L // 3)], H=1, seed=L)
    check(c, 3, L // 10)


@pytest.mark.parametrize("L", [700, 40000])
@pytest.mark.parametrize("how", ["equal", "zero", "two", "negative", "odd", "close"])
def test_weights_that_are_alike_or_odd(gpu, how, L):
    c = Evictable([L, 90], [L // 2, 33], H=2, part=L // 2 + 7, seed=3)
    rng = np.random.default_rng(5)
    w = c.weights
    if how == "equal":
        w[:] = 0.25
    elif how == "zero":
        w[:] = 0.0
        w[rng.random(w.shape) < 0.5] = -0.0
    elif how == "two":
        w[:] = np.where(rng.random(w.shape) < 0.3, 1.5, 0.125)
    elif how == "negative":
        w[:] = rng.standard_normal(w.shape)
    elif how == "odd":
        w[:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.0],
                                   np.float32), w.shape)
    else:                                # differ in their last bits alone
        w[:] = (np.float32(1.0).view(np.uint32) + rng.integers(0, 40, w.shape, np.uint32)
                ).view(np.float32)
    check(c, 1, 5, how)


def test_sequences_left_alone_beside_others(gpu):
    c = Evictable([100, 120, 90], [30, 30, 30], H=2, part=64, seed=4)
    c.into[1] = -1
    c.keep[1] = -7                       # not looked at
    got = check(c, 2, 3, max_keep=30)
    assert got[6] == 0


def test_what_lies_around_the_kept_tokens_stays(gpu):
    # a larger reservation, its pages full of something
    c = Evictable([100, 70], [37, 20], H=2, room=[9, 4], dst_begin=1000, seed=5)
    rng = np.random.default_rng(1)
    for p in c.page_ids:
        held = (c.k_pool[p] != 0x7FC0) & (c.k_pool[p] != 0x7F)
        c.k_pool[p] = np.where(held, c.k_pool[p], rng.integers(0, 1 << 14, c.k_pool[p].shape))
    c.v_pool[c.v_pool == 0x7F] = 0x1234
    check(c, 2, 9)


def test_pages_of_one_scale_keep_their_codes(gpu):
    c = Evictable([320], [64], H=1, fp8=True, seed=6)
    c.k_scale[~np.isnan(c.k_scale)] = 0.5
    got = check(c, 3, 20)
    assert (got[4][c.page_ids[20:24]] == 0.5).all()


def test_codes_that_are_nan_stay_nan(gpu):
    c = Evictable([200], [70], H=2, fp8=True, seed=7)
    rng = np.random.default_rng(2)
    for pool in (c.k_pool, c.v_pool):
        at = rng.random(pool.shape) < 0.02
        pool[at] = rng.choice(np.array([0x7F, 0xFF], np.uint8), at.sum())
    check(c, 3, 20)


def test_repeated_evictions_between_two_routes(gpu):
    """What an eviction leaves is the next one's cache: the routes change places."""
    import torch
    c = Evictable([200, 90], [128, 64], H=2, fp8=True, part=1 << 30, seed=8)
    first = check(c, 4, 16)
    k, v, w, routes, ks, vs, _ = first
    c.k_pool, c.v_pool, c.weights, c.routes, c.k_scale, c.v_scale = k, v, w, routes, ks, vs
    c.into = c.seq_route_begin[:-1].copy()
    c.keep = np.array([100, 3], np.int32)
    got = check(c, 4, 16)
    assert got[6] == 0 and (got[3][c.into, 3] - got[3][c.into, 2] == [100, 3]).all()


@pytest.mark.parametrize("what", ["into", "before", "other", "full", "keep", "negative", "csr", "row",
                                  "cap", "base", "page", "dst_page", "end"])
def test_refusals_leave_the_sequence_as_it_was(gpu, what):
    c = Evictable([100, 150, 80], [40, 50, 30], H=2, part=64, seed=9)
    row = int(c.seq_route_begin[1])
    to = int(c.into[1])
    flag, max_keep = 2, 50
    if what == "into":
        c.into[1] = len(c.routes)
    elif what == "before":
        c.into[1] = -2
    elif what == "other":
        c.into[1] = c.into[0]
    elif what == "full":
        c.into[1] = row
    elif what == "keep":
        c.keep[1] = 51
    elif what == "negative":
        c.keep[1] = -1
    elif what == "csr":
        c.seq_route_begin[2] = len(c.routes) + 1      # the third row is bad with it
    elif what == "row":
        c.routes[row, 0] = 0
    elif what == "cap":
        c.routes[to, 5] = 3
        flag = 1
    elif what == "base":
        c.routes[to, 4] = len(c.page_ids) - 3
    elif what == "page":
        c.page_ids[c.routes[row, 4] + 1] = -1
        flag = 4
    elif what == "dst_page":
        c.page_ids[c.routes[to, 4] + 3] = c.k_pool.shape[0]
        flag = 4
    else:
        c.routes[to, 2:4] = 2 ** 31 - 20
    got = check(c, 4, 10, max_keep=max_keep)
    assert got[6] == flag
    assert np.array_equal(got[3][row], c.routes[row])
    if what != "csr":
        assert got[3][c.into[0] if what != "other" else c.seq_route_begin[1] - 1][3] == 40


def test_more_routes_than_a_call_takes(gpu):
    c = Evictable([1030 * 2, 40], [50, 20], H=1, part=2, seed=10)
    got = check(c, 1, 4)
    assert got[6] == 2
    c = Evictable([1023 * 2, 40], [50, 20], H=1, part=2, seed=10)
    assert check(c, 1, 4)[6] == 0


def test_many_sequences(gpu):
    rng = np.random.default_rng(0)
    lens = [int(x) for x in rng.integers(0, 90, 300)]
    c = Evictable(lens, [int(x) for x in rng.integers(0, 60, 300)], H=1, part=32, seed=11)
    check(c, 2, 5)


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(gpu, seed):
    rng = np.random.default_rng(300 + seed)
    B = int(rng.integers(1, 7))
    lens = [int(x) for x in rng.integers(0, 900, B)]
    c = Evictable(lens, [int(x) for x in rng.integers(0, 500, B)], H=int(rng.integers(1, 4)),
                  fp8=bool(rng.integers(2)), part=int(rng.choice([7, 50, 200, 1 << 30])),
                  first=[int(x) for x in rng.integers(-100, 100, B)], seed=seed)
    check(c, int(rng.choice([0, 1, 4, 100])), int(rng.choice([0, 3, 40, 300])),
          head_major=bool(rng.integers(2)), G=int(rng.integers(1, 17)))


def test_graph_replays_and_streams(gpu):
    import torch
    c = Evictable([300, 1, 77, 640], [100, 5, 40, 333], H=2, fp8=True, part=112, seed=1)
    want = evict_oracle(c, 4, 20)
    call, w, d = evict_gpu(c, 4, 20, run=False)
    start = {k: (w if k == "w" else d[k]).clone() for k in ("w", "routes", "k_pool", "v_pool",
                                                            "k_scale", "v_scale")}

    def reset():
        for k, t in start.items():
            (w if k == "w" else d[k]).copy_(t)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert_evicted(evict_result(c, d, w), want, "stream")
    reset()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        reset()
        (torch.ones(1 << 16, device="cuda") * i).sum().item()
        g.replay()
        torch.cuda.synchronize()
        assert_evicted(evict_result(c, d, w), want, f"replay {i}")


@pytest.mark.parametrize("fp8", [False, True])
def test_one_long_sequence_among_short_ones(gpu, fp8):
    # a long one, where the launch has a workgroup per sequence
    lens = [40000] + [20] * 9
    c = Evictable(lens, [7000] + [15] * 9, H=1, fp8=fp8, part=9000, seed=12)
    check(c, 4, 500)


@pytest.mark.parametrize("L", [8191, 8192, 8193, 16385, 32767, 32768, 32769, 65535, 65536, 65537])
@pytest.mark.parametrize("part", [70000, 1000])
def test_lengths_around_what_one_workgroup_holds(gpu, L, part):
    c = Evictable([L] + [20] * 9, [L // 4] + [15] * 9, H=1, part=part, seed=L)
    c.weights[np.random.default_rng(3).random(c.weights.shape) < 0.3] = 0.5
    check(c, 4, L // 8)


@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (9000, 0, 9000), (20000, 20000, 0),
                                             (30000, 10, 10), (25000, 0, 1), (70000, 5, 5),
                                             (0, 0, 0)])
def test_parts_of_a_long_sequence(gpu, keep, first, last):
    c = Evictable([30000, 9000], [keep, keep], H=2, part=7000, seed=13)
    c.weights[np.random.default_rng(3).random(c.weights.shape) < 0.4] = 0.5
    check(c, first, last)


@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (9000, 0, 9000), (20000, 20000, 0),
                                             (60000, 10, 10), (100000, 5, 5), (0, 0, 0)])
@pytest.mark.parametrize("fp8", [False, True])
def test_parts_of_longer_sequences(gpu, keep, first, last, fp8):
    c = Evictable([80000, 30000], [keep, keep], H=1, fp8=fp8, part=17000, seed=13)
    c.weights[np.random.default_rng(3).random(c.weights.shape) < 0.4] = 0.5
    check(c, first, last)


@pytest.mark.parametrize("what", ["page", "first_page", "dst_page", "cap", "row"])
def test_refusals_of_a_long_sequence(gpu, what):
    c = Evictable([30000, 20000], [900, 1000], H=2, part=7000, seed=14)
    row, to = int(c.seq_route_begin[1]), int(c.into[1])
    bad = 1
    if what == "page":
        c.page_ids[c.routes[row + 2, 4] + 300] = -1
    elif what == "first_page":           # behind them: the first one that takes what stays
        c.page_ids[c.routes[row + 2, 4] + 400] = -1
        bad = 0
    elif what == "dst_page":
        c.page_ids[c.routes[to, 4] + 60] = c.k_pool.shape[0]
    elif what == "cap":
        c.routes[to, 5] = 3
    else:
        c.routes[row, 0] = 0
    got = check(c, 4, 10)
    assert got[6] == {"page": 4, "first_page": 4, "dst_page": 4, "cap": 1, "row": 2}[what]
    lo, hi = c.seq_route_begin[bad], c.seq_route_begin[bad + 1]
    assert np.array_equal(got[3][lo:hi], c.routes[lo:hi])
    assert got[3][c.into[1 - bad], 3] == (900, 1000)[1 - bad]


@pytest.mark.parametrize("what", ["page", "first_page", "dst_page", "cap", "row"])
def test_refusals_of_longer_sequences(gpu, what):
    """The same where several workgroups tell a sequence's tokens apart."""
    c = Evictable([70000, 40000], [900, 1000], H=2, part=17500, seed=14)
    row, into = int(c.seq_route_begin[1]), [int(x) for x in c.into]
    bad = 0 if what == "first_page" else 1
    if what == "page":
        c.page_ids[c.routes[row + 1, 4] + 1000] = -1
    elif what == "first_page":           # the first one that sequence 0's tokens go to
        c.page_ids[c.routes[into[0], 4]] = -1
    elif what == "dst_page":
        c.page_ids[c.routes[into[1], 4] + 60] = c.k_pool.shape[0]
    elif what == "cap":
        c.routes[into[1], 5] = 3
    else:
        c.routes[row, 0] = 0
    got = check(c, 4, 10)
    assert got[6] == {"page": 4, "first_page": 4, "dst_page": 4, "cap": 1, "row": 2}[what]
    lo, hi = c.seq_route_begin[bad], c.seq_route_begin[bad + 1]
    assert np.array_equal(got[3][lo:hi], c.routes[lo:hi])
    assert got[3][into[1 - bad], 3] == (900, 1000)[1 - bad]


@pytest.mark.parametrize("how", ["short", "end"])
@pytest.mark.parametrize("long", [False, True])
def test_a_full_target_at_the_end_of_the_page_table_is_full(gpu, how, long):
    """Too few pages reserved is a full tail wherever the route lies: also where the pages
    that it lacks (or the tokens' places) would be beyond the table."""
    c = (Evictable([70000, 40000], [900, 1000], H=2, part=17500, seed=14) if long else
         Evictable([100, 150], [40, 50], H=2, part=64, seed=9))
    to = int(c.into[1])
    assert (evict_parts(c) > 1) == long
    c.routes[to, 5] -= 1
    if how == "short":                   # the last reservation ends with the table
        c.page_ids = c.page_ids[:c.routes[to, 4] + c.routes[to, 5]]
    else:
        c.routes[to, 2:4] = 2 ** 31 - 20
    lo = int(c.seq_route_begin[1])
    got = check(c, 4, 10)
    assert got[6] == 1 and np.array_equal(got[3][lo:], c.routes[lo:])
    assert got[3][c.into[0], 3] == c.keep[0]


@pytest.mark.parametrize("long", [False, True])
def test_what_stays_is_a_route_that_the_bounds_of_the_call_hold(gpu, long):
    """More pages of tokens than max_pages_per_route would be a bad route to every call
    behind the eviction: refused, and the sequence as it was."""
    c = (Evictable([70000, 40000], [900, 17000], H=2, part=16384, seed=14) if long else
         Evictable([100, 150, 80], [40, 50, 30], H=2, part=32, seed=9))
    c.max_pages = 1024 if long else 3
    assert (evict_parts(c) > 1) == long
    lo, hi = c.seq_route_begin[1:3]
    got = check(c, 4, 10)
    assert got[6] == 2 and np.array_equal(got[3][lo:hi], c.routes[lo:hi])
    assert all(got[3][c.into[b], 3] == c.keep[b] for b in range(len(c.lens)) if b != 1)


@pytest.mark.parametrize("how", ["equal", "zero", "two", "negative", "odd", "close"])
def test_weights_that_are_alike_or_odd_in_several_parts(gpu, how):
    """Told apart by several workgroups, beside a sequence left alone, short ones and an
    empty one."""
    c = Evictable([120000, 120000, 9000, 700, 0], [9000, 9, 3000, 300, 5], H=1, part=17000, seed=3)
    c.into[1] = -1
    assert evict_parts(c) > 1
    rng = np.random.default_rng(5)
    w = c.weights
    if how == "equal":
        w[:] = 0.25
    elif how == "zero":
        w[:] = 0.0
        w[rng.random(w.shape) < 0.5] = -0.0
    elif how == "two":
        w[:] = np.where(rng.random(w.shape) < 0.05, 1.5, 0.125)
    elif how == "negative":
        w[:] = rng.standard_normal(w.shape)
    elif how == "odd":
        w[:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 3.0],
                                   np.float32), w.shape)
    else:                                # differ in their last bits alone
        w[:] = (np.float32(1.0).view(np.uint32) + rng.integers(0, 40, w.shape, np.uint32)
                ).view(np.float32)
    got = check(c, 1, 5, how)
    assert got[6] == 0


@pytest.mark.parametrize("L", [8191, 8192, 8193, 40000, 65536, 65537])
def test_lengths_in_several_parts(gpu, L):
    """Around the parts' own edges, beside a sequence that makes the mean a long one."""
    c = Evictable([L, 200000], [L // 3, 100], H=1, part=1000, seed=L)
    c.weights[np.random.default_rng(3).random(c.weights.shape) < 0.3] = 0.5
    assert evict_parts(c) > 1
    check(c, 4, L // 8)


@pytest.mark.parametrize("what", ["equal", "nan", "all", "none", "edges"])
def test_where_the_threshold_lies_in_several_parts(gpu, what):
    """None or all of what competes stays; ties over every part; wanted ones that end at a
    part's edge."""
    L = 131072
    keep = {"all": L, "none": 1200, "edges": 4 + 1000 + 16384}.get(what, 20000)
    c = Evictable([L], [keep], H=2, part=30000, seed=5)
    assert evict_parts(c) > 1
    if what == "nan":
        c.weights[:] = np.nan
    elif what != "all":
        c.weights[:] = 0.5
    if what == "none":
        check(c, 200, 1000)
    else:
        check(c, 4, 1000)
