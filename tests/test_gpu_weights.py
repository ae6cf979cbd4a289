"""kf_attn_weights against the fp64 oracle, elementwise within the bounds that its
32-bit sums give (budget_testlib.assert_weights)."""
import numpy as np
import pytest

from budget_testlib import (assert_weights, rows_lse, start_weights, weights_gpu, weights_oracle,
                            weights_segments)
from rows_testlib import Cache, Rows

pytestmark = pytest.mark.gpu


def check(r, decay=0.7, what="", lse=None, **kw):
    w = start_weights(r.cache)
    lse = rows_lse(r) if lse is None else lse
    got = weights_gpu(r, lse, w, decay, **kw)
    assert_weights(got, weights_oracle(r, lse, w, decay), w, what)
    return got


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 7, 8, 16])
def test_every_group_size(gpu, G, fp8):
    lens = [70, 1, 33, 200]
    c = Cache(lens, H=2, fp8=fp8, part=64, seed=G)
    check(Rows(c, lens, G, seed=G), what=f"G {G}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 15, 16, 17, 18, 33, 64, 65, 100])
def test_every_number_of_rows(gpu, rows, fp8):
    c = Cache([300, 129], H=2, fp8=fp8, part=100, seed=rows)
    check(Rows(c, [rows, 1], 4, seed=rows), what=f"rows {rows}")


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_whole_prompts_of_every_length(gpu, n):
    c = Cache([n], H=1, seed=n)
    check(Rows(c, [n], 4, seed=n), what=f"n {n}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("decay", [0.0, 1.0, 0.5, -1.0])
def test_decays(gpu, decay, fp8):
    c = Cache([500, 40, 260], H=2, fp8=fp8, part=128, spare=2, seed=4)
    for counts in ([1, 1, 1], [32, 40, 200]):
        check(Rows(c, counts, 4, seed=5), decay)


def test_nothing_is_read_with_a_decay_of_zero(gpu):
    c = Cache([200, 90], H=2, seed=4)
    for counts in ([1, 1], [30, 90]):
        r = Rows(c, counts, 4, seed=5)
        lse, w = rows_lse(r), start_weights(c)
        nan = np.full_like(w, np.nan)
        got, clean = weights_gpu(r, lse, nan, 0.0)[0], weights_gpu(r, lse, w, 0.0)[0]
        held = ~np.isnan(got)
        assert held.sum() == 290 * 2 and np.array_equal(got[held], clean[held])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_chunks_behind_a_cached_prefix(gpu, fp8, head_major):
    lens, counts = [700, 129, 64, 1025, 5], [3, 129, 1, 40, 5]
    c = Cache(lens, H=3, fp8=fp8, part=192, seed=5)
    check(Rows(c, counts, 4, seed=6), head_major=head_major, pad=24)


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_steps(gpu, fp8):
    lens = [5000, 1, 17, 900, 3000, 1024]
    c = Cache(lens, H=2, fp8=fp8, part=2000, seed=7)
    check(Rows(c, [1] * 6, 8, seed=7), 1.0)


def test_positions_before_between_and_behind_the_routes(gpu):
    c = Cache([100, 0, 50, 80, 0], H=2, part=48, first=[40, 0, 0, 1000, 7], seed=3)
    check(Rows(c, [60, 4, 0, 33, 0], 3, first_pos=[10, 0, 0, 990, 0], seed=4))
    check(Rows(c, [6, 4, 0, 3, 0], 3, first_pos=[1000, 50, 0, 5000, 0], seed=4))


def test_positions_at_the_ends_of_32_bits(gpu):
    top = 2 ** 31 - 1
    c = Cache([70, 40, 40], H=1, first=[top - 70, top - 40, -20], seed=8)
    check(Rows(c, [70, 8, 9], 2, first_pos=[top - 70, top - 3, -25], seed=8))
    check(Rows(c, [1, 1, 1], 2, first_pos=[top, top, -2 ** 31], seed=8))


@pytest.mark.parametrize("rows", [1, 40])
def test_rows_without_a_softmax_give_nothing(gpu, rows):
    c = Cache([90, 100], H=2, seed=6)
    r = Rows(c, [rows, rows], 3, seed=6)
    lse = rows_lse(r)
    lse[0, 1], lse[rows // 2, 4], lse[rows, 2], lse[-1, 0] = -np.inf, np.nan, np.nan, np.inf
    got = check(r, lse=lse)
    assert not np.isnan(got[0]).any()


@pytest.mark.parametrize("rows", [1, 60])
def test_hidden_tokens_get_nothing_whatever_they_hold(gpu, rows):
    c = Cache([150], H=2, part=96, seed=11)
    r = Rows(c, [rows], 4, first_pos=[40], seed=11)
    lse = rows_lse(r)
    for t in (100, 110, 149):
        pid, slot = c.at(0, t)
        c.k_pool[pid, :, slot] = 0x7F80 if t == 110 else 0x7FC0
    got = check(r, lse=lse)
    assert not np.isnan(got[0]).any()
    pid, slot = c.at(0, 110)
    assert (got[0][pid, :, slot] == 0.0).all()


@pytest.mark.parametrize("scale", [0.0, -0.2])
@pytest.mark.parametrize("rows", [2, 50])
def test_scales(gpu, scale, rows):
    c = Cache([150], H=2, seed=1)
    r = Rows(c, [rows], 4, seed=2)
    lse, w = rows_lse(r, scale), start_weights(c)
    # (a scale 2.3 times the usual one: so many times the error of a score)
    got, ref = weights_gpu(r, lse, w, 1.0, scale), weights_oracle(r, lse, w, 1.0, scale)
    assert got[1] == ref[1] == 0
    assert np.all(np.abs(got[0] - ref[0]) <= (3e-4 + ref[2] * 2.0 ** -24) * np.abs(ref[0]) + 1e-6)


@pytest.mark.parametrize("rows", [1, 30])
def test_bad_pages_and_routes(gpu, rows):
    c = Cache([320, 100, 90, 64], H=2, part=160, seed=12)
    r = Rows(c, [rows] * 4, 4, seed=12)
    lse = rows_lse(r)
    c.page_ids[8] = c.k_pool.shape[0]
    got = check(r, lse=lse)
    assert got[1] == 4
    c.page_ids[3] = -1
    c.routes[c.seq_route_begin[1], 0] = 9          # a sequence that is not there
    c.routes[c.seq_route_begin[2], 5] = 1          # more tokens than pages
    got = check(r, lse=lse)
    assert got[1] == 6


def test_a_bad_row_of_the_row_table(gpu):
    c = Cache([40, 50, 60], H=1, seed=2)
    r = Rows(c, [10, 10, 10], 2, seed=2)
    lse = rows_lse(r)
    r.row_begin = np.array([0, 10, 5, 40], np.int32)
    got = check(r, lse=lse)
    assert got[1] == 2


def test_a_route_of_nearly_all_of_32_bits_is_refused(gpu):
    """Longer than any place behind its last token can be counted: left as it was."""
    import torch
    from paper_2606_29207_amd import kf
    pages = 2 ** 27
    ids = torch.zeros(pages, dtype=torch.int32, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    shape = kf.make_shape(1, 4, 1, kf.KV_BF16, 2, pages, 0.1)
    k = torch.zeros((2, 1, 16, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda")
    for end in (2 ** 31 - 1024, 2 ** 31 - 1):
        w, err = torch.full((2, 1, 16), 0.25, device="cuda"), torch.zeros(1, **i32)
        kf.attn_weights(shape, q, torch.zeros((1, 4), device="cuda"), torch.tensor([end - 1], **i32),
                        k, torch.tensor([[0, 0, 0, end, 0, pages]], **i32), pages, ids,
                        torch.tensor([0, 1], **i32), 1.0, w, err)
        assert (w == 0.25).all() and int(err.item()) == kf.EFLAG_BAD_ROUTE


def test_sequences_without_rows_are_not_looked_at(gpu):
    c = Cache([90, 100, 110], H=2, part=64, seed=13)
    r = Rows(c, [0, 30, 0], 2, seed=13)
    lse = rows_lse(r)
    c.routes[0, 5] = 0
    got = check(r, lse=lse)
    assert got[1] == 0


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(gpu, seed):
    rng = np.random.default_rng(200 + seed)
    B = int(rng.integers(1, 9))
    lens = [int(x) for x in rng.integers(0, 700, B)]
    counts = [int(min(n, rng.choice([0, 1, 2, 17, 100, 300]))) for n in lens]
    G, H = int(rng.integers(1, 17)), int(rng.integers(1, 4))
    c = Cache(lens, H=H, fp8=bool(rng.integers(2)), part=int(rng.choice([16, 50, 200, 1 << 30])),
              spare=int(rng.integers(3)), first=[int(x) for x in rng.integers(-100, 100, B)], seed=seed)
    check(Rows(c, counts, G, seed=seed), float(rng.choice([0.0, 0.9, 1.0])),
          head_major=bool(rng.integers(2)), pad=int(rng.choice([0, 8])))


def test_large_launches_of_every_division_of_keys(gpu):
    # enough pages that waves lie beside each other along the keys, by two and by four
    for lens in ([9000] * 2, [20000] * 2):
        c = Cache(lens, H=16, seed=5)
        check(Rows(c, [70, 1], 1, seed=5))


def test_same_bits_graph_replays_and_streams(gpu):
    import torch
    c = Cache([900, 300, 64, 2000], H=2, part=256, seed=3)
    r = Rows(c, [1, 40, 3, 130], 4, seed=3)
    lse, w0 = rows_lse(r), start_weights(c)
    want = weights_gpu(r, lse, w0, 0.5)[0]
    twice = weights_gpu(r, lse, want, 0.5)[0]
    call, w, err = weights_gpu(r, lse, w0, 0.5, run=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert np.array_equal(w.cpu().numpy(), want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    start = torch.from_numpy(w0).cuda()
    for i in range(4):
        w.copy_(start)
        (torch.ones(1 << 16, device="cuda") * i).sum().item()
        g.replay()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(w.cpu().numpy(), twice), i
    assert err.item() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_many_columns_over_stretches_of_32_pages(gpu, fp8):
    # a mean of 133 columns: workgroups of 32 pages, which the one sequence of more than
    # 256 columns takes 16 at a time
    c = Cache([2000, 900, 300, 40], H=2, fp8=fp8, seed=3)
    r = Rows(c, [130, 1, 1, 1], 4, seed=5)
    assert weights_segments(r, chunk_pages=32) == 1
    check(r)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,segments", [(70, 2), (96, 3), (128, 4), (160, 5), (192, 6), (224, 7),
                                           (256, 8), (400, 8)])
def test_every_number_of_segments(gpu, rows, segments, fp8):
    c = Cache([700], H=2, fp8=fp8, part=300, seed=rows)
    r = Rows(c, [rows], 4, seed=rows)
    assert weights_segments(r) == segments
    check(r)


@pytest.mark.parametrize("spare,segments", [(550, 1), (1300, 1), (260, 4)])
def test_long_prompts_of_many_routes(gpu, spare, segments):
    # so many workgroups that each takes all columns of its keys, or four share them
    c = Cache([300, 310, 290], H=2, part=32, spare=spare, seed=spare)
    r = Rows(c, [300, 280, 100], 4, seed=3)
    assert weights_segments(r) == segments
    check(r)


@pytest.mark.parametrize("rows", [1, 100, 600])
def test_stretches_that_a_launch_s_limit_makes_longer(gpu, rows):
    # 18 stretches of 16 pages, 16 KV heads and 60002 routes would be more than 2^24
    # workgroups: twice as many pages each
    c = Cache([600, 0], H=16, part=320, seed=4)
    n, k = 60000, len(c.page_ids)
    c.routes = np.concatenate([c.routes, np.tile(np.array([[1, 9, 0, 0, k, 0]], np.int32), (n, 1))])
    c.page_ids = np.concatenate([c.page_ids, np.full(288 - k, -1, np.int32)])
    c.max_pages = 288
    r = Rows(c, [rows, 0], 1, first_pos=[600 - rows, 0], seed=rows)
    w = start_weights(c)
    lse = (4.0 + np.random.default_rng(1).random((rows, 16))).astype(np.float32)
    got = weights_gpu(r, lse, w, 0.7)
    assert_weights(got, weights_oracle(r, lse, w, 0.7), w)


@pytest.mark.parametrize("rows", [1, 40, 100])
def test_sequences_that_share_pages_in_calls_of_their_own(gpu, rows):
    """A prefix of 96 tokens in the routes of two sequences: each has its rows in a call
    of its own, the second one's with decay = 1."""
    c = Cache([250, 250], H=2, part=96, seed=4)
    a, b = c.seq_route_begin[:2]
    c.routes[b, 4] = c.routes[a, 4]
    w, ref = start_weights(c), start_weights(c).astype(np.float64)
    before = np.abs(w)
    flags = terms = 0
    for k, decay in ((0, 0.5), (1, 1.0)):
        r = Rows(c, [rows * (k == 0), rows * (k == 1)], 4, first_pos=[250 - rows] * 2, seed=k)
        lse = rows_lse(r)
        ref, flags, n = weights_oracle(r, lse, ref, decay)
        terms += n
        w, got = weights_gpu(r, lse, w, decay)
        assert got == flags == 0
    assert_weights((w, 0), (ref, 0, terms), before)
