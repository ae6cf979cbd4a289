"""kf_prompt_attn and kf_tree_attn against the fp64 oracle, elementwise within
bounds derived from their roundings (rows_testlib.assert_rows)."""
import numpy as np
import pytest

from rows_testlib import DIM, Cache, Rows, assert_rows, bits

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------- prompts
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 16])
def test_prompts_of_every_group_size(gpu, G, fp8):
    lens = [70, 1, 33, 200]
    c = Cache(lens, H=2, fp8=fp8, part=64, seed=G)
    r = Rows(c, lens, G, seed=G)
    assert_rows(r.gpu(), r.oracle(), f"G {G}")


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_whole_prompts_of_every_length(gpu, n):
    c = Cache([n], H=1, seed=n)
    r = Rows(c, [n], 4, seed=n)
    assert_rows(r.gpu(), r.oracle(), f"n {n}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
def test_chunks_behind_a_cached_prefix(gpu, fp8, head_major):
    lens, counts = [700, 129, 64, 1025, 5], [3, 129, 1, 40, 5]
    c = Cache(lens, H=3, fp8=fp8, part=192, seed=5)
    r = Rows(c, counts, 4, seed=6)
    assert_rows(r.gpu(head_major=head_major, pad=24), r.oracle())


def test_sequences_without_rows_and_rows_without_tokens(gpu):
    # positions before the first token (a node that holds a later range), between
    # routes and behind the last one; sequences of no rows and of no tokens
    c = Cache([100, 0, 50, 80, 0], H=2, part=48, first=[40, 0, 0, 1000, 7], seed=3)
    r = Rows(c, [60, 4, 0, 33, 0], 3, first_pos=[10, 0, 0, 990, 0], seed=4)
    got, ref = r.gpu(), r.oracle()
    assert np.isneginf(ref[1]).sum() > 0
    assert_rows(got, ref)


def test_positions_at_the_ends_of_32_bits(gpu):
    top = 2 ** 31 - 1
    c = Cache([70, 40, 40], H=1, first=[top - 70, top - 40, -20], seed=8)
    r = Rows(c, [70, 8, 9], 2, first_pos=[top - 70, top - 3, -25], seed=8)
    assert_rows(r.gpu(), r.oracle())


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.5])
def test_scales(gpu, scale):
    c = Cache([150], H=2, seed=1)
    r = Rows(c, [150], 4, seed=2)
    got, ref = r.gpu(scale), r.oracle(scale)
    # scores of scale 1.5 reach 60: their products' sums are off by 17 times more
    wide = max(1.0, abs(scale) / 0.0884)
    d = np.abs(got[1] - ref[1])
    assert d.max() <= 1e-4 * wide
    bound = 2.0 ** -8 * np.abs(ref[0]) + (2.0 ** -8 + 2.0 ** -16 + 4e-4 * (wide > 1)) * ref[3]
    assert np.all(np.abs(got[0] - ref[0]) <= bound + 1e-30)


@pytest.mark.parametrize("fp8", [False, True])
def test_few_rows_over_a_long_cache_are_split(gpu, fp8):
    c = Cache([9000, 20, 4096], H=2, fp8=fp8, part=4096, seed=9)
    r = Rows(c, [4, 20, 1], 4, seed=9)
    assert_rows(r.gpu(), r.oracle())


def test_rows_of_no_sequence_are_left_alone(gpu):
    c = Cache([40, 30], H=1, seed=2)
    r = Rows(c, [40, 30], 2, seed=2)
    whole = r.gpu()
    extra = bits(np.random.default_rng(0).standard_normal((5, 2, DIM)))
    r.q = np.concatenate([extra[:2], r.q, extra[2:]])
    r.row_begin = r.row_begin + 2
    out, lse, flags = r.gpu()
    assert flags == 0
    assert np.array_equal(out[2:72], whole[0]) and np.array_equal(lse[2:72], whole[1])
    for x in (out, lse):
        assert np.isnan(x[:2]).all() and np.isnan(x[72:]).all()


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("H", [2, 1500])
def test_rows_without_any_sequence(gpu, tree, H):
    c = Cache([], H=H)
    r = Rows(c, [], 1, tree=tree)
    r.q = bits(np.random.default_rng(0).standard_normal((3, H, DIM)))
    if tree:
        r.k_draft, r.v_draft, r.tree_mask = r.q, r.q, np.zeros(3, np.int64)
    out, lse, flags = r.gpu()
    assert flags == 0 and np.isnan(out).all() and np.isnan(lse).all()


def test_hidden_tokens_never_reach_a_row(gpu):
    """Infinities and NaN in tokens that a row does not see: same bits."""
    n = 150
    c = Cache([n], H=2, part=96, seed=11)
    r = Rows(c, [n], 4, seed=11)
    clean = r.gpu()
    for t, v in ((100, 0x7F80), (101, 0x7FC0), (103, 0xFF80), (149, 0x7FC0)):
        pid, slot = c.at(0, t)
        c.k_pool[pid, :, slot] = 0x7FC0
        c.v_pool[pid, :, ::3, slot] = v
    out, lse, flags = r.gpu()
    assert flags == 0
    # rows up to 95 share no tile with them but the pages' own: bit for bit
    assert np.array_equal(out[:64], clean[0][:64]) and np.array_equal(lse[:64], clean[1][:64])
    # in their tile the products are added token by token: within the roundings
    ref = r.oracle()
    assert_rows((out[:100], lse[:100], 0), (ref[0][:100], ref[1][:100], 0, ref[3][:100]))
    assert np.isnan(out[100:]).all() and np.isnan(lse[100:]).all()


def test_an_infinite_value_reaches_exactly_the_rows_that_see_it(gpu):
    n = 90
    c = Cache([n], H=1, seed=12)
    r = Rows(c, [n], 2, seed=12)
    pid, slot = c.at(0, 70)
    c.v_pool[pid, 0, 5, slot] = 0x7F80
    out, lse, flags = r.gpu()
    ref = r.oracle()
    assert flags == 0 and np.isinf(ref[0][70:, :, 5]).all()
    assert np.array_equal(np.isinf(out), np.isinf(ref[0]))
    fine = np.isfinite(ref[0])
    assert (np.abs(out - ref[0])[fine] <= (2.0 ** -7 + 2.0 ** -16) * ref[3][fine]).all()


# ------------------------------------------------------------------- trees
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 8, 16])
def test_trees_of_every_group_size(gpu, G, fp8):
    lens, counts = [300, 17, 0, 64, 1000], [7, 1, 5, 64, 33]
    c = Cache(lens, H=2, fp8=fp8, part=256, seed=G)
    r = Rows(c, counts, G, tree=True, seed=G)
    assert_rows(r.gpu(), r.oracle(), f"G {G}")


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64])
def test_trees_of_every_size(gpu, n):
    c = Cache([100], H=1, seed=n)
    r = Rows(c, [n], 4, tree=True, seed=n)
    assert_rows(r.gpu(pad=8), r.oracle(), f"n {n}")


def test_masks_that_leave_rows_empty(gpu):
    """Rows of empty masks, of bits past the tree, without their own bit, of bit 63;
    over empty and short caches."""
    c = Cache([0, 3, 0], H=2, seed=1)
    r = Rows(c, [64, 4, 3], 4, tree=True, seed=1)
    m = r.tree_mask
    m[:] = np.where(np.arange(len(m)) % 3 == 0, 0, m)
    m[5] = -1                       # every bit
    m[7] = np.int64(-2 ** 63)       # the last drafted row alone
    m[64:68] = [0, 1 << 40, 2, -16]
    m[68:] = [0, 0, 0]
    got, ref = r.gpu(), r.oracle()
    assert np.isneginf(ref[1][68:]).all()
    assert_rows(got, ref)


@pytest.mark.parametrize("fp8", [False, True])
def test_trees_over_long_caches_are_split(gpu, fp8):
    c = Cache([5000, 12000, 100], H=2, fp8=fp8, part=4096, seed=4)
    r = Rows(c, [9, 16, 2], 4, tree=True, seed=4)
    assert_rows(r.gpu(head_major=True), r.oracle())


def test_hidden_drafts_never_reach_a_row(gpu):
    c = Cache([40], H=1, seed=5)
    r = Rows(c, [12], 4, tree=True, seed=5)
    r.tree_mask[:] = [1 << i for i in range(12)]      # each itself alone
    r.v_draft[3], r.k_draft[3] = 0x7F80, 0x7FC0
    r.v_draft[8, :, ::2] = 0x7FC0
    out, lse, flags = r.gpu()
    keep = [i for i in range(12) if i not in (3, 8)]
    ref = r.oracle()
    assert flags == 0
    assert_rows((out[keep], lse[keep], 0), (ref[0][keep], ref[1][keep], 0, ref[3][keep]))
    assert np.isnan(out[3]).all() and np.isnan(lse[3]).all()


# ------------------------------------------------------------- bad tables
def test_bad_pages_reach_the_rows_that_see_them(gpu):
    for bad in (-1, 1 << 30):
        c = Cache([200, 100], H=2, part=128, seed=6)
        r = Rows(c, [200, 100], 3, seed=6)
        c.page_ids[4] = bad                    # tokens 64 .. 79 of sequence 0
        got, ref = r.gpu(), r.oracle()
        assert ref[2] == 4 and np.isnan(ref[0][64:200]).all() and not np.isnan(ref[0][:64]).any()
        assert_rows(got, ref)
        t = Rows(c, [4, 6], 3, tree=True, seed=7)
        assert_rows(t.gpu(), t.oracle())


def test_bad_pages_that_no_row_sees_raise_nothing(gpu):
    c = Cache([200], H=1, seed=6)
    r = Rows(c, [40], 4, first_pos=[10], seed=6)
    c.page_ids[4:] = -5                        # tokens 64 and on; the rows reach 49
    got, ref = r.gpu(), r.oracle()
    assert ref[2] == 0
    assert_rows(got, ref)


@pytest.mark.parametrize("what", ["seq", "order", "base", "cap", "ids", "most", "csr", "csr_end"])
def test_bad_routes_reach_their_sequence(gpu, what, spare=0):
    """(spare: so many empty sequences more)"""
    c = Cache([100, 90, 60] + [0] * spare, H=1, part=64, seed=2)
    r = Rows(c, [20, 30, 10] + [0] * spare, 2, seed=2)
    row = c.routes[2]                          # sequence 1
    if what == "seq":
        row[0] = 0
    elif what == "order":
        row[3] = row[2] - 1
    elif what == "base":
        row[4] = -1
    elif what == "cap":
        row[5] = 2
    elif what == "ids":
        row[4] = len(c.page_ids) - 2
    elif what == "most":
        c.max_pages = 3
    elif what == "csr":
        c.seq_route_begin[1] = 5
    else:
        c.seq_route_begin[3] = 100 + spare
    got, ref = r.gpu(), r.oracle()
    assert ref[2] == 2 and np.isnan(ref[0]).any()
    assert_rows(got, ref, what)


@pytest.mark.parametrize("begin", [[0, 50, 20, 60], [-1, 20, 50, 60], [0, 20, 50, 61]])
def test_a_bad_row_table_makes_every_row_nan(gpu, begin):
    c = Cache([100, 90, 60], H=2, seed=2)
    for tree in (False, True):
        r = Rows(c, [20, 30, 10], 2, tree=tree, seed=2)
        r.row_begin = np.array(begin, np.int32)
        out, lse, flags = r.gpu()
        assert flags == 2 and np.isnan(out).all() and np.isnan(lse).all()


def test_too_many_drafts_of_one_sequence(gpu):
    c = Cache([30, 30], H=1, seed=2)
    r = Rows(c, [65, 64], 2, tree=True, seed=2)
    got, ref = r.gpu(), r.oracle()
    assert ref[2] == 2
    assert_rows(got, ref)


# ----------------------------------------------------------- many sequences
@pytest.mark.parametrize("B", [64, 65, 1024, 1025, 3000])
@pytest.mark.parametrize("tree", [False, True])
def test_many_sequences(gpu, B, tree):
    """Launches that find their tiles themselves (up to 64 sequences) and planned
    ones, in LDS (up to 1024) and beyond; sequences without rows, bad ones among
    them."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 60, B)
    counts = np.minimum(rng.integers(0, 4, B), lens if not tree else 64)
    c = Cache(lens, H=1, part=32, seed=B)
    r = Rows(c, counts, 2, tree=tree, seed=B)
    for b in (3, B // 2, B - 1):
        counts[b] = max(counts[b], 1)
    c.routes[c.seq_route_begin[B // 2]][4] = -3
    c.page_ids[c.routes[-1][4]:][:1] = 1 << 20
    assert_rows(r.gpu(), r.oracle(), f"B {B}")


@pytest.mark.parametrize("what", ["seq", "order", "base", "cap", "ids", "most", "csr", "csr_end"])
def test_bad_routes_of_planned_launches(gpu, what):
    test_bad_routes_reach_their_sequence(gpu, what, spare=70)


@pytest.mark.parametrize("begin", [[0, 50, 20, 60], [-1, 20, 50, 60], [0, 20, 50, 61]])
def test_a_bad_row_table_of_planned_launches(gpu, begin):
    c = Cache([100, 90, 60] + [0] * 70, H=2, seed=2)
    for tree in (False, True):
        r = Rows(c, [20, 30, 10] + [0] * 70, 2, tree=tree, seed=2)
        r.row_begin = np.array(begin + begin[-1:] * 70, np.int32)
        out, lse, flags = r.gpu()
        assert flags == 2 and np.isnan(out).all() and np.isnan(lse).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_planned_splits(gpu, fp8, tree):
    """70 sequences, some long: tiles in parts of different sizes, bad routes and
    pages among split sequences."""
    lens = [5000, 20, 0, 2500, 900] + [40] * 65
    counts = [9, 20, 3 * tree, 33, 4] + [1] * 65
    c = Cache(lens, H=2, fp8=fp8, part=2048, seed=4)
    r = Rows(c, counts, 4, tree=tree, seed=4)
    assert_rows(r.gpu(), r.oracle())
    c.page_ids[c.routes[1][4] + 5] = -9        # sequence 0, token 2128 on
    c.routes[c.seq_route_begin[3] + 1][5] = 0  # sequence 3
    ref = r.oracle()
    assert ref[2] == 6
    assert_rows(r.gpu(), ref)


@pytest.mark.parametrize("B,rows,n,tree,fp8", [
    (10, 1, 1600, True, False), (10, 2, 1600, False, True), (5, 1, 3200, True, True),
    (5, 130, 1750, False, False)])
def test_equal_tiles_in_a_shorter_last_round(gpu, B, rows, n, tree, fp8):
    """Tiles of one length that fill no whole rounds of the workgroups (64 KV heads, so
    that a round has few): those of the last one are split."""
    c = Cache([n] * B, H=64, fp8=fp8, part=1500, seed=B)
    r = Rows(c, [rows] * B, 1, tree=tree, seed=rows)
    assert_rows(r.gpu(), r.oracle())
    if rows < 100:
        c.page_ids[c.routes[3][4] + 1] = -1       # sequence 1, second route
        c.routes[2 * B - 2][4] = -1               # the last sequence
        ref = r.oracle()
        assert ref[2] == 6
        assert_rows(r.gpu(), ref)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(gpu, seed):
    """Drawn batches: with a plan and without, split and whole, several routes that a
    row sees all of, in part or not at all."""
    rng = np.random.default_rng(100 + seed)
    tree, fp8 = bool(seed & 1), bool(seed & 2)
    B = int(rng.choice([1, 3, 20, 64, 70, 130]))
    H, G = int(rng.integers(1, 4)), int(rng.choice([1, 2, 3, 4, 5, 8]))
    lens = np.exp(rng.uniform(0, np.log([60, 400, 6000][int(rng.integers(3))]), B)).astype(int)
    lens[rng.random(B) < 0.1] = 0
    lens[rng.integers(B)] += int(rng.integers(0, 5000))
    counts = np.exp(rng.uniform(0, np.log(64), B)).astype(int)
    counts[rng.random(B) < 0.1] = 0
    budget = 300_000   # (row, token) pairs that the oracle works through
    while (counts * (lens + 1)).sum() > budget:
        counts //= 2
    c = Cache(lens, H=H, fp8=fp8, part=int(rng.choice([16, 48, 500, 1 << 20])), seed=seed,
              first=rng.integers(0, 3, B) * 32)
    first_pos = [int(rng.integers(-2, n + 70)) for n in lens]
    r = Rows(c, counts, G, tree=tree, first_pos=first_pos, seed=seed)
    if seed % 3 == 0 and tree:
        r.tree_mask = rng.integers(-2 ** 63, 2 ** 63 - 1, len(r.tree_mask))  # any bits
    assert_rows(r.gpu(head_major=bool(seed & 4)), r.oracle(), f"seed {seed}")


# ------------------------------------------------------------ how it is run
def test_same_bits_for_any_placement_stream_and_repeat(gpu):
    import torch
    lens, counts = [3000, 500, 77], [5, 64, 30]
    for tree in (False, True):
        c = Cache(lens, H=2, part=1024, seed=3)
        r = Rows(c, counts, 4, tree=tree, seed=3)
        a = r.gpu()
        b = r.gpu(stream=torch.cuda.Stream())
        d = r.gpu(head_major=True, pad=8)
        for x in (b, d):
            assert np.array_equal(a[0], x[0]) and np.array_equal(a[1], x[1])


@pytest.mark.parametrize("tree", [False, True])
def test_graph_replays(gpu, tree):
    """A captured call replayed with other queries between eager work."""
    import torch
    c = Cache([4000, 300], H=2, part=2048, seed=3)
    r = Rows(c, [8, 20], 4, tree=tree, seed=3)
    call, out, lse, err = r.gpu(run=False)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    q = call._keep[1]
    for k in range(4):
        q.copy_(torch.randn(q.shape, device="cuda").to(torch.bfloat16))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        a, b = out.clone(), lse.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, lse), k
    assert int(err.item()) == 0


@pytest.mark.parametrize("tree", [False, True])
def test_graph_replays_of_planned_launches(gpu, tree):
    """The plan is made anew at every replay: the routes grow and the rows move
    between sequences."""
    import torch
    lens, counts = [5000, 900, 40] + [30] * 67, [4, 20, 0] + [1] * 67
    c = Cache(lens, H=2, part=2048, seed=3)
    r = Rows(c, counts, 4, tree=tree, seed=3)
    # the long sequence begins short: its last route's tokens come later
    last = c.seq_route_begin[1] - 1
    ends = [int(c.routes[last][2]) + n for n in (5, 300, 900, 904)]
    call, out, lse, err = r.gpu(run=False)
    routes, begin = call._keep[6], call._keep[9]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.synchronize()
    for k, end in enumerate(ends):
        c.routes[last][3] = end
        routes[last, 3] = end
        r.row_begin[1] = 4 + k
        begin[1] = 4 + k
        if not tree:
            r.first_pos[0] = end - 4 - k
            call._keep[-1].copy_(torch.from_numpy(r.first_pos))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        a, b = out.clone(), lse.clone()
        assert_rows((a.double().cpu().numpy(), b.double().cpu().numpy(), int(err.item())),
                    r.oracle(), f"replay {k}")
        out.fill_(float("nan"))
        call()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, lse), k


@pytest.mark.parametrize("B", [700, 1100])      # the plan's tables in LDS, in memory
@pytest.mark.parametrize("tree", [False, True])
def test_same_bits_of_tiles_in_a_shorter_last_round(gpu, tree, B):
    """Tiles of one length, more than a round of the workgroups: which of them are
    split, and so rounded in another order, follows from the arguments alone."""
    import torch
    from paper_2606_29207_amd import kf
    G, n, pages, rows = 4, 1600, 3000, 4
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)

    def normal(*size):
        return torch.randn(size, generator=gen, device="cuda").to(torch.bfloat16)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    k_pool, v_pool = normal(pages, 1, 16, DIM), normal(pages, 1, DIM, 16)
    page_ids = torch.randint(0, pages, (B * n // 16,), generator=gen, device="cuda").to(torch.int32)
    routes = ints([[b, 0, 0, n, b * n // 16, n // 16] for b in range(B)])
    q, kd, vd = normal(B * rows, G, DIM), normal(B * rows, 1, DIM), normal(B * rows, 1, DIM)
    shape = kf.make_shape(B, G, 1, kf.KV_BF16, pages, B * n // 16, DIM ** -0.5)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = None
    for k in range(12):
        out = torch.full((B * rows, G, DIM), float("nan"), dtype=torch.bfloat16, device="cuda")
        lse = torch.full((B * rows, G), float("nan"), device="cuda")
        tail = (k_pool, v_pool, routes, n // 16, page_ids, ints(range(B + 1)),
                ints([rows * b for b in range(B + 1)]), out, lse,
                kf.alloc_rows_workspace(shape, B * rows), err)
        if tree:
            kf.tree_attn(shape, q, kd, vd, torch.full((B * rows,), 15, device="cuda"), *tail)
        else:
            kf.prompt_attn(shape, q, ints([n - rows] * B), *tail)
        torch.cuda.synchronize()
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), k
    assert int(err.item()) == 0 and not out.isnan().any()


# ------------------------------------------------- exceptional values over fp8
@pytest.mark.parametrize("scale", [0.0, -0.2, 1.5])
def test_scales_over_fp8_pages(gpu, scale):
    c = Cache([150], H=2, fp8=True, seed=1)
    r = Rows(c, [150], 4, seed=2)
    got, ref = r.gpu(scale), r.oracle(scale)
    wide = max(1.0, abs(scale) / 0.0884)       # as test_scales
    assert np.abs(got[1] - ref[1]).max() <= 1e-4 * wide
    bound = 2.0 ** -8 * np.abs(ref[0]) + (2.0 ** -8 + 2.0 ** -16 + 4e-4 * (wide > 1)) * ref[3]
    assert np.all(np.abs(got[0] - ref[0]) <= bound + 1e-30)


def test_hidden_fp8_tokens_never_reach_a_row(gpu):
    n = 150
    c = Cache([n], H=2, fp8=True, part=96, seed=11)
    r = Rows(c, [n], 4, seed=11)
    clean = r.gpu()
    for t in (100, 101, 103, 149):
        pid, slot = c.at(0, t)
        c.k_pool[pid, :, slot] = 0x7F
        c.v_pool[pid, :, ::3, slot] = 0xFF
    out, lse, flags = r.gpu()
    ref = r.oracle()
    assert flags == 0 and not np.isnan(ref[0][:100]).any()
    # rows up to 95 share no tile with them
    assert np.array_equal(out[:64], clean[0][:64]) and np.array_equal(lse[:64], clean[1][:64])
    assert_rows((out[:100], lse[:100], 0), (ref[0][:100], ref[1][:100], 0, ref[3][:100]))
    assert np.isnan(out[100:]).all() and np.isnan(lse[100:]).all()


@pytest.mark.parametrize("G", [1, 3, 4])
def test_fp8_nan_values_reach_exactly_the_rows_that_see_them(gpu, G):
    """NaN codes in single dims of V: those dims of the rows that see the token, no
    other output; the page's V scale stays in the others."""
    n = 170
    c = Cache([n, 40], H=2, fp8=True, part=112, seed=13)
    r = Rows(c, [n, 40], G, seed=13)
    for t, dims, code in ((70, [5, 77], 0x7F), (71, [127], 0xFF), (75, [0], 0x7F), (130, [64], 0x7F)):
        pid, slot = c.at(0, t)
        c.v_pool[pid, 0, dims, slot] = code
    ref = r.oracle()
    assert np.isnan(ref[0][70:170, :G, 5]).all() and not np.isnan(ref[0][:70]).any()
    assert not np.isnan(ref[0][:, G:]).any() and not np.isnan(ref[1]).any()
    assert_rows(r.gpu(), ref)


def test_drafts_that_are_not_finite_over_fp8_pages(gpu):
    """Hidden ones never reach a row; a visible infinity reaches its dims of exactly
    the rows that see it."""
    c = Cache([45], H=2, fp8=True, seed=5)
    r = Rows(c, [40], 4, tree=True, seed=5)
    m = r.tree_mask
    m[:] = [1 << i for i in range(40)]         # each itself alone
    m[20:24] |= 1 << 10
    r.v_draft[3], r.k_draft[3] = 0x7F80, 0x7FC0
    r.v_draft[35, :, ::2] = 0x7FC0
    r.v_draft[10, :, 9] = 0x7F80
    r.v_draft[10, :, 40] = 0xFF80
    got, ref = r.gpu(), r.oracle()
    sees_inf = [10, 20, 21, 22, 23]
    assert np.isposinf(ref[0][sees_inf, :, 9]).all() and np.isneginf(ref[0][sees_inf, :, 40]).all()
    for sign in (np.isposinf, np.isneginf):
        assert np.array_equal(sign(got[0]), sign(ref[0]))
    assert np.isnan(got[0][3]).all() and np.isnan(got[1][3]).all()
    # the rest within its bound (infinities taken out on both sides)
    out, want, spread = (np.where(np.isinf(ref[0]), 0.0, x) for x in (got[0], ref[0], ref[3]))
    assert_rows((out, got[1], got[2]), (want, *ref[1:3], spread))


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("k, v", [(0.0, 1.0), (-1.0, 1.0), (1.0, 0.0), (1.0, -1.0), (-1.0, -2.0),
                                  (0.0, 0.0)])
def test_fp8_page_scales_of_zero_and_below(gpu, tree, k, v):
    """Such pages among ordinary ones, beside one in their tile and alone in it."""
    lens = [200, 33, 90]
    c = Cache(lens, H=2, fp8=True, part=112, seed=21)
    for b, t in ((0, 20), (0, 130), (1, 32), (2, 10), (2, 17), (2, 89)):
        pid = c.at(b, t)[0]
        c.k_scale[pid] *= np.float32(k)
        c.v_scale[pid, 1] *= np.float32(v)
    r = Rows(c, [20, 33, 30] if tree else lens, 4, tree=tree, seed=22)
    assert_rows(r.gpu(), r.oracle())


@pytest.mark.parametrize("which", ["k_scale", "v_scale"])
def test_a_nan_page_scale_reaches_the_rows_that_see_the_page(gpu, which):
    n = 120
    c = Cache([n], H=2, fp8=True, seed=23)
    getattr(c, which)[c.at(0, 80)[0], 1] = np.nan      # tokens 80 .. 95, the second of a tile's pages
    r = Rows(c, [n], 2, seed=24)
    ref = r.oracle()
    assert np.isnan(ref[0][80:, 2:]).all() and not np.isnan(ref[0][:80]).any()
    assert_rows(r.gpu(), ref)


# -------------------------------------- many sequences, bad ones that rows see
@pytest.mark.parametrize("B", [64, 65, 1024, 1025, 3000])
@pytest.mark.parametrize("tree", [False, True])
def test_many_sequences_with_bad_ones_that_have_rows(gpu, B, tree):
    rng = np.random.default_rng(B)
    lens, counts = rng.integers(0, 60, B), rng.integers(0, 4, B)
    marked = [3, B // 2, B - 1]
    lens[marked], counts[marked] = [40, 50, 37], [1, 3, 2]
    if not tree:
        counts = np.minimum(counts, lens)
    c = Cache(lens, H=1, part=32, seed=B)
    r = Rows(c, counts, 2, tree=tree, seed=B)
    c.routes[c.seq_route_begin[B // 2]][4] = -3
    c.page_ids[c.routes[-1][4]] = 1 << 20              # of the last sequence's last route
    ref = r.oracle()
    assert ref[2] == 6
    begin = r.row_begin
    for b, bad in ((3, False), (B // 2, True), (B - 1, True)):
        assert np.isnan(ref[0][begin[b]:begin[b + 1]]).all() == bad
    assert_rows(r.gpu(), ref, f"B {B}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("B", [1025, 2500])
@pytest.mark.parametrize("tree", [False, True])
def test_splits_among_more_sequences_than_the_plan_keeps_in_lds(gpu, tree, B, fp8):
    """Few rows over long sequences among a thousand that have none or are short."""
    lens, counts = np.full(B, 3), np.zeros(B, int)
    counts[::40] = 1
    for b, n, rows in ((7, 4000, 1), (B // 3, 6000, 2), (B // 2, 2500, 30), (B - 2, 5000, 2), (B - 1, 700, 1)):
        lens[b], counts[b] = n, rows
    c = Cache(lens, H=2, fp8=fp8, part=2048, seed=B)
    r = Rows(c, counts, 4, tree=tree, seed=B)
    assert_rows(r.gpu(), r.oracle())
    c.page_ids[c.routes[c.seq_route_begin[7]][4] + 9] = -1
    c.routes[c.seq_route_begin[B - 2] + 1][5] = 0
    ref = r.oracle()
    assert ref[2] == 6
    assert_rows(r.gpu(), ref)


# ------------------------------------------------- pages reserved, but not held
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("tree", [False, True])
def test_few_tokens_in_large_reservations(gpu, tree, fp8):
    """Launches cut for reserved pages, most of whose parts see no token; as many
    parts as one sequence gets, and bad tables among them."""
    for lens, counts, spare in (([40], [8], 2000), ([700, 1, 0], [5, 1, 2], 700), ([64], [64], 500),
                                ([9, 400, 3, 33], [9, 20, 3, 1], 100), ([5000], [3], 1)):
        c = Cache(lens, H=2, fp8=fp8, part=2048, spare=spare, seed=spare)
        if not tree:
            counts = np.minimum(counts, np.maximum(lens, 1))
        r = Rows(c, counts, 4, tree=tree, seed=spare)
        assert_rows(r.gpu(), r.oracle(), f"{lens}")
        if lens[0] == 9:
            c.page_ids[c.routes[1][4] + 3] = -1
            c.routes[2][5] = 0
            ref = r.oracle()
            assert ref[2] == 6
            assert_rows(r.gpu(), ref)


@pytest.mark.parametrize("part", [16, 20])
@pytest.mark.parametrize("tree", [False, True])
def test_planned_splits_of_short_routes(gpu, tree, part):
    """A tile or two a route, in plans of LDS and of memory; empty routes between."""
    for B in (70, 1030):
        lens = [2000, 1, 700, 0, 1500] + [3] * (B - 5)
        counts = [9, 1, 40, 2 * tree, 3] + [0, 1] * ((B - 5) // 2) + [0] * ((B - 5) % 2)
        c = Cache(lens, H=2, part=part, seed=B)
        c.routes[9][3] = c.routes[9][2]            # sequence 0 holds a gap
        r = Rows(c, counts, 4, tree=tree, seed=B)
        assert_rows(r.gpu(), r.oracle(), f"B {B}")
