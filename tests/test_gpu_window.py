"""kf_window_attn against the fp64 oracle, elementwise within the bounds that its
roundings give (rows_testlib.assert_rows)."""
import numpy as np
import pytest

from budget_testlib import window_gpu, window_oracle
from rows_testlib import DIM, Cache, Rows, assert_rows, bits

pytestmark = pytest.mark.gpu


def check(r, sinks, window, what="", **kw):
    assert_rows(window_gpu(r, sinks, window, **kw), window_oracle(r, sinks, window), what)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 16])
def test_every_group_size(gpu, G, fp8):
    lens = [170, 1, 33, 260]
    c = Cache(lens, H=2, fp8=fp8, part=64, seed=G)
    check(Rows(c, lens, G, seed=G), 5, 37, f"G {G}")


@pytest.mark.parametrize("sinks,window", [
    (0, 0), (0, 1), (0, 2), (1, 0), (4, 0), (3, 17), (16, 16), (17, 31), (32, 32), (33, 33),
    (64, 1), (100, 50), (0, 300), (299, 1), (300, 0), (1000, 7), (0, 2 ** 31 - 1),
    (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("fp8", [False, True])
def test_sinks_and_windows(gpu, sinks, window, fp8):
    c = Cache([300, 45], H=1, fp8=fp8, part=112, seed=3)
    check(Rows(c, [300, 45], 4, seed=4), sinks, window)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_every_length(gpu, n):
    c = Cache([n], H=1, seed=n)
    check(Rows(c, [n], 4, seed=n), 2, 20, f"n {n}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_chunks_behind_a_cached_prefix(gpu, fp8, head_major):
    lens, counts = [700, 129, 64, 1025, 5], [3, 129, 1, 40, 5]
    c = Cache(lens, H=3, fp8=fp8, part=192, seed=5)
    check(Rows(c, counts, 4, seed=6), 10, 130, head_major=head_major, pad=24)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 100, 1000])
def test_decode_steps(gpu, fp8, window):
    lens = [5000, 1, 17, 900, 3000, 1024]
    c = Cache(lens, H=2, fp8=fp8, part=1024, seed=7)
    check(Rows(c, [1] * 6, 4, seed=7), 4, window)


@pytest.mark.parametrize("B,part", [(70, 1 << 30), (130, 48), (1100, 100)])
def test_many_sequences(gpu, B, part):
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(0, 400, B)]
    counts = [min(n, int(x)) for n, x in zip(lens, rng.choice([0, 1, 1, 3, 40], B))]
    c = Cache(lens, H=1, part=part, seed=B)
    check(Rows(c, counts, 2, seed=B), 3, 90)


@pytest.mark.parametrize("fp8", [False, True])
def test_planned_splits(gpu, fp8):
    # few long row tiles among many short ones: their keys are split
    lens = [9000, 40] * 2 + [60] * 66
    counts = [60, 1] * 2 + [2] * 66
    c = Cache(lens, H=2, fp8=fp8, part=2048, seed=9)
    check(Rows(c, counts, 4, seed=9), 40, 6000)


def test_routes_out_of_order_and_with_gaps(gpu):
    c = Cache([300, 200], H=2, part=80, first=[20, -60], seed=3)
    for b in range(2):     # a sequence's routes in the table's order, not the tokens'
        a, e = c.seq_route_begin[b], c.seq_route_begin[b + 1]
        c.routes[a:e] = c.routes[a:e][::-1].copy()
        c.routes[a:a + 1, 2:4] += 500
    r = Rows(c, [50, 60], 3, first_pos=[290, 100], seed=4)
    for sinks, window in ((30, 100), (0, 64), (150, 0), (90, 700)):
        check(r, sinks, window, f"{sinks} {window}")


def test_rows_without_tokens_and_sequences_without_rows(gpu):
    c = Cache([100, 0, 50, 80, 0], H=2, part=48, first=[40, 0, 0, 1000, 7], seed=3)
    r = Rows(c, [60, 4, 0, 33, 0], 3, first_pos=[10, 0, 0, 990, 0], seed=4)
    ref = window_oracle(r, 3, 9)
    assert np.isneginf(ref[1]).sum() > 0
    assert_rows(window_gpu(r, 3, 9), ref)
    # a window that lies behind every token
    r = Rows(c, [6, 4, 0, 3, 0], 3, first_pos=[1000, 50, 0, 5000, 0], seed=4)
    ref = window_oracle(r, 0, 100)
    assert np.isneginf(ref[1]).all()
    assert_rows(window_gpu(r, 0, 100), ref)


def test_positions_at_the_ends_of_32_bits(gpu):
    top = 2 ** 31 - 1
    c = Cache([70, 40, 40, 50], H=1, first=[top - 70, top - 40, -20, -2 ** 31], seed=8)
    r = Rows(c, [70, 8, 9, 20], 2, first_pos=[top - 70, top - 3, -25, -2 ** 31], seed=8)
    for sinks, window in ((0, 10), (5, 33), (top, 0), (0, top), (7, 1)):
        check(r, sinks, window, f"{sinks} {window}")


@pytest.mark.parametrize("fp8", [False, True])
def test_tokens_outside_the_window_never_reach_a_row(gpu, fp8):
    """Infinities and NaN in what no row sees, or only some do."""
    n = 200
    c = Cache([n], H=2, fp8=fp8, part=96, seed=11)
    r = Rows(c, [100], 4, seed=11)
    for t, v in ((50, 0x7FC0), (64, 0x7F80), (65, 0xFF80), (70, 0x7FC0)):
        pid, slot = c.at(0, t)
        c.k_pool[pid, :, slot] = 0x7F if fp8 else 0x7FC0
        c.v_pool[pid, :, ::3, slot] = 0x7F if fp8 else v
    # rows 100 .. 199, window 40: tokens 61 .. 199 and sinks 0 .. 9
    got, ref = window_gpu(r, 10, 40), window_oracle(r, 10, 40)
    clean = slice(10, 100)              # from position 110 on none of them is seen
    assert not np.isnan(got[0][clean]).any() and not np.isnan(ref[0][clean]).any()
    assert_rows((got[0][clean], got[1][clean], 0), (ref[0][clean], ref[1][clean], 0, ref[3][clean]))
    sees = [i for i in range(10) if 100 + i - 40 < 70]
    assert np.isnan(got[0][sees]).all() and np.isnan(got[1][sees]).all()


def test_bad_pages_reach_the_rows_that_see_them(gpu):
    c = Cache([320], H=2, seed=12)
    r = Rows(c, [200], 2, seed=12)
    c.page_ids[8] = c.k_pool.shape[0]          # tokens 128 .. 143
    check(r, 4, 30)
    c.page_ids[0] = -5                          # the sinks' page
    check(r, 4, 30)


def test_bad_pages_that_no_row_sees_raise_nothing(gpu):
    c = Cache([320], H=2, seed=12)
    r = Rows(c, [100], 2, seed=12)
    c.page_ids[5] = 1 << 30
    ref = window_oracle(r, 4, 60)
    assert ref[2] == 0
    assert_rows(window_gpu(r, 4, 60), ref)


@pytest.mark.parametrize("what", ["seq", "order", "cap", "base", "pages"])
def test_bad_routes_reach_their_sequence(gpu, what):
    c = Cache([90, 100, 110], H=1, part=64, seed=13)
    r = Rows(c, [20, 30, 40], 2, seed=13)
    row = int(c.seq_route_begin[1])
    col, v = {"seq": (0, 2), "order": (3, -1), "cap": (5, 1), "base": (4, -1),
              "pages": (3, 16 * 40)}[what]
    c.routes[row, col] = v
    ref = window_oracle(r, 2, 25)
    assert ref[2] and np.isnan(ref[0][20:50]).all()
    assert_rows(window_gpu(r, 2, 25), ref)


@pytest.mark.parametrize("begin", [[0, 5, 3, 20], [-1, 2, 3, 4], [0, 5, 9, 21]])
def test_a_bad_row_table_makes_every_row_nan(gpu, begin):
    c = Cache([30, 30, 30], H=1, seed=2)
    r = Rows(c, [5, 5, 10], 2, seed=2)
    r.row_begin = np.array(begin, np.int32)
    out, lse, flags = window_gpu(r, 1, 9)
    assert flags == 2 and np.isnan(out).all() and np.isnan(lse).all()


def test_rows_of_no_sequence_are_left_alone(gpu):
    c = Cache([40, 30], H=1, seed=2)
    r = Rows(c, [40, 30], 2, seed=2)
    whole = window_gpu(r, 2, 11)
    extra = bits(np.random.default_rng(0).standard_normal((5, 2, DIM)))
    r.q = np.concatenate([extra[:2], r.q, extra[2:]])
    r.row_begin = r.row_begin + 2
    out, lse, flags = window_gpu(r, 2, 11)
    assert flags == 0
    assert np.array_equal(out[2:72], whole[0]) and np.array_equal(lse[2:72], whole[1])
    for x in (out, lse):
        assert np.isnan(x[:2]).all() and np.isnan(x[72:]).all()


def test_a_window_over_everything_is_a_prompt(gpu):
    c = Cache([150, 40], H=2, part=64, seed=5)
    r = Rows(c, [150, 7], 4, seed=5)
    a, b = window_gpu(r, 0, 1000), r.gpu()
    assert a[2] == b[2] == 0
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(gpu, seed):
    rng = np.random.default_rng(100 + seed)
    B = int(rng.integers(1, 9))
    lens = [int(x) for x in rng.integers(0, 700, B)]
    counts = [int(min(n, rng.choice([0, 1, 2, 17, 100, 300]))) for n in lens]
    G, H = int(rng.integers(1, 17)), int(rng.integers(1, 4))
    c = Cache(lens, H=H, fp8=bool(rng.integers(2)), part=int(rng.choice([16, 50, 200, 1 << 30])),
              spare=int(rng.integers(3)), first=[int(x) for x in rng.integers(-100, 100, B)], seed=seed)
    r = Rows(c, counts, G, seed=seed)
    check(r, int(rng.choice([0, 1, 5, 64, 200])), int(rng.choice([0, 1, 16, 47, 300, 5000])),
          head_major=bool(rng.integers(2)), pad=int(rng.choice([0, 8])))


def test_graph_replays_and_streams(gpu):
    import torch
    c = Cache([900, 300, 64, 2000], H=2, part=256, seed=3)
    r = Rows(c, [1, 40, 3, 130], 4, seed=3)
    want = window_gpu(r, 4, 200)
    d = c.device()
    call, out, lse, err = window_gpu(r, 4, 200, d=d, run=False)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), want[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        (torch.ones(1 << 16, device="cuda") * i).sum().item()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.double().cpu().numpy(), want[0]), i
        assert np.array_equal(lse.double().cpu().numpy(), want[1]), i
    assert err.item() == 0
