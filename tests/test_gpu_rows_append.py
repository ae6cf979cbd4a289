"""kf_kv_append_rows: bit for bit the oracle's pools, scales, routes and flags,
and bit for bit what one kf_kv_append per token leaves."""
import numpy as np
import pytest

import oracle
from rows_testlib import DIM, Cache, bits

pytestmark = pytest.mark.gpu


def _rows(n, H, seed, spread=1.0):
    """Rows whose sizes differ by up to `spread` (fp8 pages are then re-encoded)."""
    rng = np.random.default_rng(seed)
    size = np.exp(rng.uniform(0, np.log(spread), (n, H, 1))) if spread > 1 else 1.0
    return tuple(bits(rng.standard_normal((n, H, DIM)) * size) for _ in range(2))


def _append(c, k, v, begin, row_list=None, head_major=False, pad=0, call=1):
    """The call's pools, scales, routes (as the oracle lays them out) and flags."""
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import _to_dev
    d = c.device(head_major)

    def wide(x):
        t = _to_dev(x, "cuda")
        if pad:
            w = torch.full((t.shape[0], c.H * DIM + pad), float("nan"), dtype=torch.bfloat16,
                           device="cuda")
            w[:, pad:] = t.reshape(t.shape[0], -1)
            t = w[:, pad:].unflatten(1, (c.H, DIM))
        return t

    bound = kf.bind_kv_append_rows(
        c.shape(c.H, head_major=head_major), d["k_pool"], d["v_pool"], wide(k), wide(v),
        d["routes"], _to_dev(np.asarray(begin, np.int32), "cuda"), d["page_ids"], d["err"],
        row_list=None if row_list is None else _to_dev(np.asarray(row_list, np.int32), "cuda"),
        k_scale=d["k_scale"], v_scale=d["v_scale"])
    for _ in range(call):
        bound()
    torch.cuda.synchronize()
    got = []
    for n in ("k_pool", "v_pool"):
        t = d[n].cpu()
        t = t.numpy() if c.fp8 else t.view(torch.int16).numpy().view(np.uint16)
        got.append(np.swapaxes(t, 0, 1) if head_major else t)
    if c.fp8:
        got += [d["k_scale"].cpu().numpy(), d["v_scale"].cpu().numpy()]
    return got + [d["routes"].cpu().numpy(), int(d["err"].item())]


def _check(c, k, v, begin, row_list=None, flags=0, **kw):
    ref = oracle.kv_append_rows(c.k_pool, c.v_pool, c.routes, c.page_ids, k, v, begin, row_list,
                                num_seqs=len(c.lens), k_scale=c.k_scale, v_scale=c.v_scale)
    got = _append(c, k, v, begin, row_list, **kw)
    assert got[-1] == ref[-1] == flags, (got[-1], ref[-1])
    for a, b, n in zip(got[:-1], ref[:-1], ("k_pool", "v_pool", "k_scale", "v_scale")
                       if c.fp8 else ("k_pool", "v_pool", "routes")):
        assert np.array_equal(a.view(np.uint32) if a.dtype == np.float32 else a,
                              b.view(np.uint32) if b.dtype == np.float32 else b), n
    assert np.array_equal(got[-2], ref[-2])
    return ref


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("H", [1, 3, 8])
def test_few_and_many_rows(gpu, H, head_major, fp8):
    lens = [0, 1, 15, 16, 17, 40, 5]
    for counts in ([1, 15, 1, 16, 33, 0, 2], [40, 100, 17, 3, 0, 300, 64]):
        c = Cache(lens, H=H, fp8=fp8, spare=25, seed=H)
        begin = np.concatenate([[0], np.cumsum(counts)])
        k, v = _rows(int(begin[-1]), H, H)
        _check(c, k, v, begin, head_major=head_major, pad=16 * (H == 3))


@pytest.mark.parametrize("n", [1, 2, 3, 15, 16, 17, 31, 32, 33, 255, 256, 257, 1000])
@pytest.mark.parametrize("fp8", [False, True])
def test_one_route_of_every_count(gpu, n, fp8):
    for start in (0, 9):
        c = Cache([start], H=2, fp8=fp8, spare=80, seed=n)
        _check(c, *_rows(n, 2, n), [0, n])


@pytest.mark.parametrize("counts", [[5, 3, 16], [300, 7, 90]])
def test_fp8_pages_are_re_encoded_within_a_call(gpu, counts):
    """Token sizes over a range of 4000: a page's scale is raised several times,
    over resident slots and over the call's own."""
    for seed in range(6):
        c = Cache([11, 3, 0], H=2, fp8=True, spare=30, seed=seed)
        begin = np.concatenate([[0], np.cumsum(counts)])
        k, v = _rows(int(begin[-1]), 2, seed, spread=4000.0)
        k[0, 0] = 0
        v[int(begin[2])] = 0                   # a first token of zeros: scale 1
        _check(c, k, v, begin)


def test_every_bf16_value_is_stored_as_single_appends_store_it(gpu):
    """All finite bf16 values through the E4M3 rule (subnormals and ties among them)."""
    allv = np.array([b for b in range(65536) if (b >> 7) & 0xFF != 0xFF], np.uint16)
    rows = np.resize(allv, (-(-len(allv) // DIM), 1, DIM))
    c = Cache([0], H=1, fp8=True, spare=40)
    _check(c, rows, rows[::-1].copy(), [0, len(rows)])


@pytest.mark.parametrize("fp8", [False, True])
def test_equal_to_single_appends(gpu, fp8):
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import _to_dev
    n, B, H = 21, 3, 2
    c = Cache([7, 0, 30], H=H, fp8=fp8, spare=4, seed=1)
    k, v = _rows(B * n, H, 3, spread=300.0)
    got = _append(c, k, v, [0, n, 2 * n, 3 * n])
    d = c.device()
    tail = torch.arange(B, dtype=torch.int32, device="cuda")
    for i in range(n):
        pick = [i, n + i, 2 * n + i]
        kf.kv_append(c.shape(H), d["k_pool"], d["v_pool"], _to_dev(k[pick], "cuda"),
                     _to_dev(v[pick], "cuda"), d["routes"], tail, d["page_ids"], d["err"],
                     k_scale=d["k_scale"], v_scale=d["v_scale"])
    torch.cuda.synchronize()
    assert int(d["err"].item()) == 0 == got[-1]
    for t, g in zip((d["k_pool"], d["v_pool"]), got):
        t = t.cpu()
        assert np.array_equal(t.numpy() if fp8 else t.view(torch.int16).numpy().view(np.uint16), g)
    assert np.array_equal(d["routes"].cpu().numpy(), got[-2])
    if fp8:
        assert np.array_equal(d["k_scale"].cpu().numpy(), got[2], equal_nan=True)
        assert np.array_equal(d["v_scale"].cpu().numpy(), got[3], equal_nan=True)


@pytest.mark.parametrize("fp8", [False, True])
def test_row_lists(gpu, fp8):
    """Rows picked in any order, some twice, some never; entries before the first
    and behind the last route's."""
    rng = np.random.default_rng(5)
    k, v = _rows(50, 2, 6)
    for counts in ([3, 0, 17, 6], [60, 200, 1, 33]):
        c = Cache([4, 9, 0, 16], H=2, fp8=fp8, spare=15, seed=2)
        begin = 2 + np.concatenate([[0], np.cumsum(counts)])
        lst = rng.integers(0, 50, int(begin[-1]) + 3)
        lst[[0, -1]] = -7, 1000                # of no route: not looked at
        _check(c, k, v, begin, lst, pad=8)


def test_a_prompt_over_two_routes_of_a_sequence(gpu):
    c = Cache([64, 10], H=2, part=32, spare=70, seed=2)
    c.routes[0][5] += 0
    k, v = _rows(700, 2, 6)
    _check(c, k, v, [0, 0, 600, 700])


@pytest.mark.parametrize("many", [False, True])
def test_a_route_takes_all_of_its_rows_or_none(gpu, many):
    n = 300 if many else 20

    def fresh():
        c = Cache([5, 6, 7], H=2, spare=n // 16 + 2, seed=4)
        return c, [0, n, 2 * n, 3 * n], list(range(3 * n))

    k, v = _rows(3 * n, 2, 1)
    for what, flags in (("full", 1), ("page", 4), ("row", 2), ("seq", 2), ("order", 2),
                        ("base", 2), ("csr", 2), ("csr_end", 2), ("far", 2)):
        c, begin, lst = fresh()
        if what == "full":
            c.routes[1][5] = (6 + n - 1) // 16
        elif what == "page":
            c.page_ids[c.routes[1][4] + 1] = c.k_pool.shape[0]
        elif what == "row":
            lst[2 * n - 1] = 3 * n
        elif what == "seq":
            c.routes[1][0] = 3
        elif what == "order":
            c.routes[1][3] = -1
        elif what == "base":
            c.routes[1][4] = len(c.page_ids) - 1
        elif what == "csr":
            begin = [0, n, n - 1, 3 * n]
        elif what == "csr_end":
            begin = [0, n, 2 * n, 3 * n + 1]
        else:
            c.routes[1][2:4] = 2 ** 31 - 10, 2 ** 31 - 4
        ref = _check(c, k, v, begin, lst, flags=flags)
        assert ref[2][0][3] == (5 if "csr" in what else 5 + n), what


# A call of up to 64 entries, at most three a route on the mean, is one launch.
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("H", [1, 3, 8])
def test_a_few_rows_for_each_of_many_routes(gpu, H, head_major, fp8):
    for seed in range(4):
        rng = np.random.default_rng(seed)
        B = int(rng.choice([1, 20, 22, 64, 500]))
        counts = rng.multinomial(min(64, 3 * B) - seed % 2, np.ones(B) / B)
        if seed == 3 and B > 1:
            counts = np.sort(counts)
            counts[-1], counts[:-1] = counts.sum(), 0      # one route takes them all
        c = Cache(rng.integers(0, 60, B), H=H, fp8=fp8, spare=6, seed=seed)
        begin = np.concatenate([[0], np.cumsum(counts)])
        n = int(begin[-1])
        k, v = _rows(2 * n, H, seed, spread=1.0 if seed < 2 else 500.0)
        _check(c, k, v, begin, rng.permutation(2 * n)[:n], head_major=head_major, pad=8 * (seed & 1))


@pytest.mark.parametrize("n", [64, 65])
def test_both_sides_of_one_launch(gpu, n):
    counts = [2] * 31 + [n - 62]
    c = Cache([14] * 32, H=2, fp8=True, spare=2, seed=n)
    _check(c, *_rows(n, 2, n, spread=50.0), np.concatenate([[0], np.cumsum(counts)]))


def test_all_or_none_in_one_launch(gpu):
    n, rest = 20, [0] * 20
    k, v = _rows(3 * n, 2, 1)
    for what, flags in (("full", 1), ("page", 4), ("row", 2), ("seq", 2), ("order", 2),
                        ("base", 2), ("csr", 2), ("far", 2)):
        c = Cache([5, 6, 7] + rest, H=2, spare=n // 16 + 2, seed=4)
        begin, lst = [0, n, 2 * n, 3 * n] + [3 * n] * 20, list(range(3 * n))
        if what == "full":
            c.routes[1][5] = (6 + n - 1) // 16
        elif what == "page":
            c.page_ids[c.routes[1][4] + 1] = c.k_pool.shape[0]
        elif what == "row":
            lst[2 * n - 1] = 3 * n
        elif what == "seq":
            c.routes[1][0] = 23
        elif what == "order":
            c.routes[1][3] = -1
        elif what == "base":
            c.routes[1][4] = len(c.page_ids) - 1
        elif what == "csr":
            begin[-1] = 3 * n + 1
        else:
            c.routes[1][2:4] = 2 ** 31 - 10, 2 ** 31 - 4
        ref = _check(c, k, v, begin, lst, flags=flags)
        assert ref[2][0][3] == (5 if what == "csr" else 5 + n), what


def test_captured_appends_of_single_rows(gpu):
    """Four replays beside four eager calls: the routes move, the pages are crossed."""
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import _to_dev
    c = Cache([13, 14, 31, 0], H=2, fp8=True, spare=4, seed=4)
    begin = _to_dev(np.arange(0, 9, 2, dtype=np.int32), "cuda")
    sides = []
    for _ in range(2):
        d = c.device()
        k, v = (_to_dev(x, "cuda") for x in _rows(8, 2, 0))
        sides.append((d, k, v, kf.bind_kv_append_rows(
            c.shape(2), d["k_pool"], d["v_pool"], k, v, d["routes"], begin, d["page_ids"], d["err"],
            k_scale=d["k_scale"], v_scale=d["v_scale"])))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        sides[1][3]()
    torch.cuda.synchronize()
    for step in range(4):
        x = _rows(8, 2, step + 1, spread=100.0)
        for d, k, v, _ in sides:
            k.copy_(_to_dev(x[0], "cuda"))
            v.copy_(_to_dev(x[1], "cuda"))
        sides[0][3]()
        graph.replay()
        torch.cuda.synchronize()
        for n in ("k_pool", "v_pool", "routes", "err", "k_scale", "v_scale"):
            a, b = (s[0][n].view(torch.int32) if s[0][n].dtype == torch.float32 else s[0][n]
                    for s in sides)
            assert torch.equal(a, b), (n, step)
    assert int(sides[0][0]["err"].item()) == 0


def test_captured_appends(gpu):
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import _to_dev
    for counts in ([3, 4], [200, 150]):
        for fp8 in (False, True):
            c = Cache([5, 30], H=2, fp8=fp8, spare=100, seed=4)
            begin = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
            sides = []
            for _ in range(2):
                d = c.device()
                k, v = (_to_dev(x, "cuda") for x in _rows(int(begin[-1]), 2, 0))
                call = kf.bind_kv_append_rows(c.shape(2), d["k_pool"], d["v_pool"], k, v, d["routes"],
                                              _to_dev(begin, "cuda"), d["page_ids"], d["err"],
                                              k_scale=d["k_scale"], v_scale=d["v_scale"])
                sides.append((d, k, v, call))
            side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
                sides[1][3]()
            torch.cuda.synchronize()
            for step in range(4):
                x = _rows(int(begin[-1]), 2, step + 1)
                for d, k, v, _ in sides:
                    k.copy_(_to_dev(x[0], "cuda"))
                    v.copy_(_to_dev(x[1], "cuda"))
                sides[0][3]()
                graph.replay()
                torch.cuda.synchronize()
                for n in ("k_pool", "v_pool", "routes", "err") + (("k_scale", "v_scale") if fp8 else ()):
                    a, b = sides[0][0][n], sides[1][0][n]
                    a, b = ((x.view(torch.int16) if x.dtype == torch.bfloat16 else
                             x.view(torch.int32) if x.dtype == torch.float32 else x) for x in (a, b))
                    assert torch.equal(a, b), (n, step)
            assert int(sides[0][0]["err"].item()) == 0


@pytest.mark.parametrize("n", [6, 21, 90])      # one launch, and planned ones
@pytest.mark.parametrize("start", [0, 9])       # a page that begins with the call, or goes on
def test_zeros_keep_their_sign(gpu, n, start):
    """-0.0 beside ordinary values, on pages whose scale stays: 0x80, as single
    appends store it; a page of zeros alone (scale 1) too."""
    import torch
    from paper_2606_29207_amd import kf
    from paper_2606_29207_amd.step import _to_dev
    H, routes = 2, 4
    rng = np.random.default_rng(n + start)
    k, v = _rows(routes * n, H, n)
    for x in (k, v):
        x[rng.random(x.shape) < 0.2] = 0x8000
        x[rng.random(x.shape) < 0.1] = 0x0000
        x[rng.random(x.shape) < 0.05] = 0x8001           # rounds to a zero of its sign
        x[-n:] = np.where(rng.random(x[-n:].shape) < 0.5, 0x8000, 0)
    begin = np.arange(routes + 1) * n
    c = Cache([start] * routes, H=H, fp8=True, spare=7, seed=n)
    c.k_scale *= 16                                      # room, as appends leave it
    c.v_scale *= 16
    ref = _check(c, k, v, begin)
    assert (ref[0] == 0x80).sum() > 100 and (ref[1] == 0x80).sum() > 100
    d = c.device()
    tail = torch.arange(routes, dtype=torch.int32, device="cuda")
    for i in range(n):
        pick = begin[:-1] + i
        kf.kv_append(c.shape(H), d["k_pool"], d["v_pool"], _to_dev(k[pick], "cuda"),
                     _to_dev(v[pick], "cuda"), d["routes"], tail, d["page_ids"], d["err"],
                     k_scale=d["k_scale"], v_scale=d["v_scale"])
    torch.cuda.synchronize()
    assert int(d["err"].item()) == 0
    assert np.array_equal(d["k_pool"].cpu().numpy(), ref[0])
    assert np.array_equal(d["v_pool"].cpu().numpy(), ref[1])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("counts", [[56, 96, 8, 0], [2, 1, 3, 2], [0, 30, 20, 60]])
def test_a_prompt_over_several_routes_of_a_sequence(gpu, counts, fp8):
    """Rows into three routes of one sequence in one call: a partly filled range, two
    empty ones behind it, and another sequence's."""
    c = Cache([200, 10], H=2, fp8=fp8, part=96, spare=5, seed=2)
    assert [list(r[:1]) for r in c.routes] == [[0], [0], [0], [1]]
    for r, end in enumerate((40, 96, 192)):
        c.routes[r][3] = end
    begin = np.concatenate([[0], np.cumsum(counts)])
    k, v = _rows(int(begin[-1]), 2, 6, spread=30.0)
    ref = _check(c, k, v, begin)
    assert list(ref[-2][:, 3]) == [40 + counts[0], 96 + counts[1], 192 + counts[2], 10 + counts[3]]


# Calls of more than 128 routes (one launch) and of more than 2048 (planned) read the
# table of entries in other ways.
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("R", [128, 129, 2048, 2049, 5000])
def test_many_routes_of_which_few_take_rows(gpu, R, fp8):
    for n, seed in ((1, 0), (64, 1), (65, 2), (400, 3), (3 * min(R, 1000), 4)):
        rng = np.random.default_rng(R + seed)
        counts = rng.multinomial(n, np.ones(R) / R)
        if seed in (1, 2):                                   # the first, the last, one of many
            counts[:] = 0
            counts[[0, R // 2, R - 1]] = 1, n - 3, 2
        c = Cache(rng.integers(0, 40, R), H=2, fp8=fp8, spare=5 + n // 16 * (seed in (1, 2)), seed=seed)
        begin = np.concatenate([[0], np.cumsum(counts)]) + (2 if n == 65 else 0)
        k, v = _rows(n + 2, 2, seed)
        _check(c, k, v, begin, rng.permutation(n + 2) if n != 400 else None)


@pytest.mark.parametrize("n", [40, 3000])
def test_all_or_none_among_many_routes(gpu, n):
    R = 2500
    k, v = _rows(n, 2, 1)
    for what, flags in (("full", 1), ("page", 4), ("row", 2), ("base", 2), ("csr", 2), ("csr_end", 2)):
        counts = np.full(R, n // R)
        counts[[0, 700, R - 1]] += 4
        counts[20] = 0
        counts = np.minimum(counts, n)
        begin = np.concatenate([[0], np.cumsum(counts)])
        lst = np.arange(max(n, int(begin[-1]))) % n
        c = Cache(np.arange(R) % 20, H=2, spare=2, seed=4)
        if what == "full":
            c.routes[700][5] = 0
        elif what == "page":
            c.page_ids[c.routes[700][4]] = -1
            c.routes[700][2:4] = 0, 3
        elif what == "row":
            lst[begin[700] + 3] = n
        elif what == "base":
            c.routes[700][4] = len(c.page_ids)
        elif what == "csr":
            begin[1000] = begin[700]
        else:
            begin[-1] = len(lst) + 1
        ref = _check(c, k, v, begin, lst, flags=flags)
        assert ref[2][0][3] == (0 if "csr" in what else begin[1]), what


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("n", [1000, 1024, 1025, 5000])
def test_one_route_among_many_takes_thousands(gpu, n, listed):
    """Checks of one route by a wave and by four; its last page and last row are looked at."""
    R, at = 2100, 1234
    c = Cache(np.arange(R) % 18, H=1, spare=1, seed=n)
    c.routes[at, 4], c.routes[at, 5] = len(c.page_ids), -(-n // 16) + 2
    pool = c.k_pool.shape[0]
    c.page_ids = np.concatenate([c.page_ids, np.arange(c.routes[at, 5]) + pool]).astype(np.int32)
    more = len(c.page_ids) - pool + 10
    c.k_pool = np.concatenate([c.k_pool, np.zeros((more, *c.k_pool.shape[1:]), np.uint16)])
    c.v_pool = np.concatenate([c.v_pool, np.zeros((more, *c.v_pool.shape[1:]), np.uint16)])
    counts = np.zeros(R, int)
    counts[[3, at]] = 2, n - 2
    begin = np.concatenate([[0], np.cumsum(counts)])
    k, v = _rows(n, 1, 1)
    lst = np.random.default_rng(n).permutation(n) if listed else None
    _check(c, k, v, begin, lst)
    end = int(c.routes[at][3] - c.routes[at][2]) + n - 2
    if listed:
        lst[-1] = n
        ref = _check(c, k, v, begin, lst, flags=2)
    else:
        c.page_ids[c.routes[at][4] + (end - 1) // 16] = -1
        ref = _check(c, k, v, begin, lst, flags=4)
    assert ref[2][3][3] == 3 + 2 and ref[2][at][3] == c.routes[at][3]
