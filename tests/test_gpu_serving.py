"""Paged serving on the GPU against plain implementations in 64 bits
(oracle/paging.py): page plans, cache writes, page copies, attention over the
cache and beam selection, alone and as one step of a beam search."""
import numpy as np
import pytest

from oracle import paging

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def serving():
    from paper_2410_13839_amd import serving as s
    return s


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a)).to(dtype).cuda()


def host(t):
    return t.detach().float().cpu().numpy() if t.dtype == torch.bfloat16 else t.detach().cpu().numpy()


def tables(rng, kv, max_pages, pages):
    """Disjoint random pages, -1 behind the last one."""
    order = rng.permutation(pages)
    t = np.full((len(kv), max_pages), -1, np.int32)
    at = 0
    for c, n in enumerate(kv):
        k = -(-int(n) // 16)
        t[c, :k] = order[at:at + k]
        at += k
    return t


# ------------------------------------------------------------------- plans
def check_plan(length, add, table, pages, max_tokens, parent=None, in_place=False):
    want = paging.plan(length, add, table, pages, max_tokens, parent)
    tb = dev(table)
    got = serving().plan_pages(dev(length), dev(add), tb, pages, max_tokens, None if parent is None else dev(parent),
                               out_table=tb if in_place else None)
    for k, w in want.items():
        assert np.array_equal(host(getattr(got, k)), w), (k, host(getattr(got, k)), w)
    return want


@pytest.mark.parametrize("n,m,hi,add_hi", [(1, 1, 0, 1), (1, 3, 20, 20), (7, 5, 60, 20), (8, 229, 3600, 4),
                                           (64, 40, 500, 130), (257, 17, 255, 17), (4096, 2, 20, 12),
                                           (256, 4, 60, 3), (200, 61, 900, 9), (70, 1000, 15000, 700)])
@pytest.mark.parametrize("beams", [False, True])
def test_plan(n, m, hi, add_hi, beams):
    rng = np.random.default_rng(n * 1000 + m)
    length = rng.integers(0, hi + 1, n)
    add = rng.integers(0, add_hi + 1, n)
    pages = n * m + 5
    table = tables(rng, length, m, pages)
    parent = np.minimum(rng.integers(0, n, n) // 4 * 4 + rng.integers(0, 4, n), n - 1) if beams else None
    if beams:
        for c in range(n):                       # full pages of a parent may be shared already
            if rng.random() < 0.3 and length[c] >= 16:
                o = rng.integers(0, n)
                k = min(length[c], length[o]) // 16
                table[c, :k] = table[o, :k]
        add = np.minimum(add, 16 * m - length[parent])
    check_plan(length, add, table, pages, int(add.sum()) + int(rng.integers(0, 40)), parent)
    if not beams:
        check_plan(length, add, table, pages, int(add.sum()), in_place=True)


@pytest.mark.parametrize("pages", [1, 15, 16, 17, 31, 32, 33, 64, 1000, 4097, 70001, 131072, 131073, 300001])
def test_plan_hands_out_the_lowest_free_pages(pages):
    rng = np.random.default_rng(pages)
    m = 40
    length = np.array([0, min(16 * (pages // 2), 16 * m), 5 if pages > 3 else 0])
    table = tables(rng, length, m, pages)
    add = np.array([3, 0, 30])
    check_plan(length, add, table, pages, 40)


def test_plan_reports_what_it_cannot_do():
    rng = np.random.default_rng(5)
    n, m, pages = 9, 6, 12
    length = np.array([17, 3, -1, 40, 16 * m, 2 ** 31 - 1, 33, 0, 5])
    table = tables(rng, np.where((length < 0) | (length > 96), 0, length) // 20, m, pages)
    table[3] = [pages, -7, 2 ** 31 - 1, 0, 0, 0]
    add = np.array([1, -1, 0, 9, 1, 0, 2 ** 31 - 1, 70, 2])
    want = check_plan(length, add, table, pages, 20)
    assert all(want["status"][1:] > 0)
    # a pool without room, rows with and without pages of their own
    want = check_plan([17, 0, 30], [40, 17, 3], np.array([[2, 0, -1, -1], [-1] * 4, [1, 4, -1, -1]]), 6, 60)
    assert want["status"].tolist() == [3, 0, 0, 0]
    parent = np.array([0, 9, -1, 3, 3, 2 ** 31 - 1, 8, 8, 0])
    want = check_plan(length, np.array([0, 0, 0, 1, 2, 1, 30, 31, 1]), table, pages, 20, parent)
    assert want["status"][1] >= 3


@pytest.mark.parametrize("n,m", [(6, 9), (40, 70), (256, 130), (300, 40)])
@pytest.mark.parametrize("beams", [False, True])
def test_plan_counts_bad_entries_of_every_row_that_keeps_them(n, m, beams):
    rng = np.random.default_rng(n + m)
    length = rng.integers(0, 16 * m - 20, n)
    pages = n * m
    table = tables(rng, length, m, pages)
    table[rng.random((n, m)) < 0.1] = -1
    table[rng.random((n, m)) < 0.1] = pages + 3
    parent = rng.integers(0, n, n) if beams else None
    add = rng.integers(0, 20, n)
    add[::7] = -1                                          # (taken as empty: no parent's children)
    want = check_plan(length, add, table, pages, 12 * n, parent)
    assert want["status"][2] > 0


# ------------------------------------------------------- writes and copies
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,D,strided", [(1, 1, 64, False), (5, 3, 64, True), (40, 2, 128, False), (333, 5, 128, True),
                                           (700, 16, 64, True)])
def test_write(dtype, T, H, D, strided):
    rng = np.random.default_rng(T)
    g = torch.Generator().manual_seed(T)
    pages = T // 16 + 9
    pool = torch.randn((pages, 2, H, 16 * D), generator=g).to(dtype)
    qkv = torch.randn((T, 3 * H * D + 8), generator=g).to(dtype)
    k, v = (qkv[:, i * H * D:(i + 1) * H * D].view(T, H, D) for i in (1, 2))
    if not strided:
        k, v = k.contiguous(), v.contiguous()
    kinds = {"runs": np.arange(T) + 5, "mixed": rng.permutation(pages * 16)[:T]}
    runs = np.concatenate([rng.permutation(T // 16 + 1)[:, None] * 16 + np.arange(16)]).reshape(-1)[:T]
    kinds["pages"] = runs
    for name, slots in kinds.items():
        slots = slots.copy()
        if T > 3:
            slots[[1, 3]] = [-1, pages * 16]     # skipped
        want = pool.float().numpy().copy()
        paging.write(want, dtype == torch.bfloat16, slots, k.float().numpy(), v.float().numpy())
        p = pool.cuda()
        qd = qkv.cuda()
        kd, vd = (qd[:, i * H * D:(i + 1) * H * D].view(T, H, D) for i in (1, 2))
        if not strided:
            kd, vd = kd.contiguous(), vd.contiguous()
        serving().write_pages(p, dev(slots), kd, vd)
        assert np.array_equal(host(p.float()), want), name


@pytest.mark.parametrize("shape,dtype", [((3, 9, 2, 1, 1024), torch.bfloat16), ((40, 2, 3, 2048), torch.float32),
                                         ((12, 70, 2, 5, 1024), torch.bfloat16)])
def test_copy(shape, dtype):
    rng = np.random.default_rng(len(shape))
    pools = torch.randn(shape, generator=torch.Generator().manual_seed(1)).to(dtype)
    pages = shape[-4]
    order = rng.permutation(pages)
    n = pages // 2 - 1
    copies = np.stack([order[:n], order[n:2 * n]], 1).astype(np.int32)
    copies = np.concatenate([copies, [[-1, -1], [order[0], -1], [-1, order[-1]], [pages, order[-1]], [order[0], pages],
                                      [order[-1], order[-1]]]]).astype(np.int32)
    want = pools.clone()
    for s, d in copies[:n]:
        want[..., d, :, :, :] = pools[..., s, :, :, :]
    got = pools.cuda()
    serving().copy_pages(got, dev(copies))
    assert torch.equal(got.cpu(), want)


# --------------------------------------------------------------- attention
WIDTH = 0                                                  # of every case's table, where it is more than the rows need


def attention_case(seed, kv, q_len, HQ, H, D, dtype, strided=False, spare=3, nan_behind=True):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    kv, q_len = np.asarray(kv), np.asarray(q_len)
    m = max(1, int(-(-kv.max() // 16))) + seed % 3
    pages = int(sum(-(-int(n) // 16) for n in kv)) + spare
    table = tables(rng, kv, max(m, WIDTH), pages)
    pool = torch.randn((pages, 2, H, 16 * D), generator=g).to(dtype)
    if nan_behind:                               # what lies behind a row's last key must not matter
        kp = pool[:, 0].view(pages, H, 16, D)
        vp = pool[:, 1].view(pages, H, D, 16) if dtype == torch.bfloat16 else pool[:, 1].view(pages, H, 16, D).transpose(2, 3)
        for c, n in enumerate(kv):
            if n % 16:
                kp[table[c, n // 16], :, n % 16:] = NAN
                vp[table[c, n // 16], :, :, n % 16:] = INF if c % 2 else NAN
    T = int(q_len.sum())
    width = HQ * D
    q = (torch.randn((T + 4, width + (24 if strided else 0)), generator=g) * 1.5).to(dtype)
    start = np.concatenate([[0], np.cumsum(q_len)]).astype(np.int32)
    return dict(pool=pool, table=table, row_start=start, kv_len=kv.astype(np.int32), q=q, T=T, HQ=HQ, D=D, strided=strided)


def run_attention(c, causal=True, window=0, scale=None, max_kv=0):
    HQ, D, T = c["HQ"], c["D"], c["T"]
    q = c["q"].cuda()
    qv = q[:, :HQ * D].view(-1, HQ, D) if c["strided"] else q[:, :HQ * D].contiguous().view(-1, HQ, D)
    buf = torch.full((T + 4, HQ * D + (16 if c["strided"] else 0)), 7.0, dtype=c["pool"].dtype, device="cuda")
    out = buf[:, :HQ * D].view(-1, HQ, D)
    got = serving().attend_pages(c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), qv,
                                 causal=causal, window=window, scale=scale, max_kv=max_kv, out=out)
    assert got is out
    return host(buf.float())


def check_attention(c, causal=True, window=0, scale=None, max_kv=0):
    """|error| <= sum p|V| (rounding of p to bf16, 2 x the scores' error, the float32 sums) + the output's rounding.
    A score is a float32 sum of D products and a scaling: within (D + 4) 2^-24 of the sum of their magnitudes, plus the
    base-2 exponential's argument, |s| log2(e) 2^-23, and its own 2^-22; sums over the keys add 64 roundings at most per
    partial sum and the partial sums' merges."""
    HQ, D, T = c["HQ"], c["D"], c["T"]
    bf = c["pool"].dtype == torch.bfloat16
    got = run_attention(c, causal, window, scale, max_kv)
    qn = c["q"].float().numpy()[:, :HQ * D].reshape(-1, HQ, D)[:T + 4]
    want = np.full((T + 4, HQ, D), 7.0)
    bound = np.zeros((2, T + 4, HQ, D))
    paging.attend(c["pool"].float().numpy(), bf, c["table"], c["row_start"], c["kv_len"], qn, want, causal, window, scale,
                  bound)
    out = got[:, :HQ * D].reshape(-1, HQ, D)
    u = 2.0 ** -24
    ds = (D + 8) * u * bound[1] + 4 * u
    tol = bound[0] * (2 * ds + 1100 * u + (2.0 ** -8 if bf else 0.0)) + np.abs(want) * (2.0 ** -8 if bf else u) + 1e-30
    assert np.isfinite(out).all()
    worst = (np.abs(out - want) / tol).max()
    assert worst <= 1.0, worst
    assert (got[T:] == 7.0).all() and (got[:, HQ * D:] == 7.0).all()      # rows behind the last, columns beside
    return worst


LENGTHS = [
    ([1], [1]), ([16], [1]), ([17], [4]), ([33], [33]), ([5, 1, 64], [5, 1, 3]),
    ([100, 0, 31, 48, 7], [1, 0, 31, 2, 7]), ([1075], [4]), ([65, 129, 200], [65, 70, 16]),
    ([513, 40, 1, 777], [1, 1, 1, 1]), ([300, 301], [257, 130]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (8, 2, 128), (7, 1, 64), (3, 3, 128), (20, 1, 128)])
@pytest.mark.parametrize("i", range(len(LENGTHS)))
def test_attention_causal(i, HQ, H, D, dtype):
    kv, q_len = LENGTHS[i]
    check_attention(attention_case(i + 10 * HQ + D, kv, q_len, HQ, H, D, dtype, strided=i % 2 == 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (12, 4, 128), (16, 1, 64)])
@pytest.mark.parametrize("kv,q_len", [([50, 0, 129], [3, 9, 140]), ([1], [70]), ([700, 16], [1, 1]), ([90, 33, 64], [64, 65, 1])])
def test_attention_full(kv, q_len, HQ, H, D, dtype):
    check_attention(attention_case(len(kv) + HQ, kv, q_len, HQ, H, D, dtype, strided=True), causal=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window", [1, 2, 16, 37, 200, 100000])
def test_attention_window(window, dtype):
    check_attention(attention_case(window, [400, 63, 700], [130, 1, 3], 4, 2, 64, dtype), window=window)
    check_attention(attention_case(window + 1, [700, 20, 90], [1, 1, 1], 8, 2, 128, dtype), window=window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q", [1, 150])
def test_attention_rows_that_see_nothing(q, dtype):
    # fewer keys than queries: the first queries of a causal row sit before position 0
    c = attention_case(3, [0, 2, 40, 7], [q, q, q, 1], 4, 2, 64, dtype)
    c["kv_len"] = np.array([0, 2, 40, -5], np.int32)
    check_attention(c)
    check_attention(c, causal=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q", [1, 4, 140])
def test_attention_pages_outside_the_pool_are_not_seen(q, dtype):
    c = attention_case(11, [200, 180, 300], [q, q, q], 4, 2, 64, dtype)
    P = c["pool"].shape[0]
    c["table"][0, 3] = -1
    c["table"][1, :] = P                                  # no page at all
    c["table"][2, [0, 5, 18]] = [2 ** 31 - 1, -2 ** 31, P]
    check_attention(c)
    check_attention(c, causal=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D,q", [(2, 2, 64, 4), (4, 1, 128, 4), (2, 2, 64, 150), (4, 2, 128, 200)])
def test_attention_what_is_not_seen_never_matters(HQ, H, D, q, dtype):
    """Infinite and NaN keys and values at positions that later queries of a chunk see and earlier ones do not: the
    earlier ones' outputs are finite and right, the later ones' are not finite."""
    n = q + 90
    c = attention_case(7, [n, n], [q, q], HQ, H, D, dtype, nan_behind=False)
    clean = attention_case(7, [n, n], [q, q], HQ, H, D, dtype, nan_behind=False)
    P = c["pool"].shape[0]
    vp = c["pool"][:, 1].view(P, H, D, 16) if dtype == torch.bfloat16 else c["pool"][:, 1].view(P, H, 16, D).transpose(2, 3)
    pos = n - 2                                           # seen by the last two queries only
    vp[c["table"][0, pos // 16], :, :, pos % 16] = INF
    vp[c["table"][1, pos // 16], :, :, pos % 16] = NAN
    a, b = run_attention(c), run_attention(clean)
    for r in range(2):
        lo, hi = r * q, (r + 1) * q
        assert np.array_equal(a[lo:hi - 2], b[lo:hi - 2])
        assert not np.isfinite(a[hi - 2:hi, :HQ * D]).any()
    # a NaN key that nobody but the last query sees
    c = attention_case(7, [n, n], [q, q], HQ, H, D, dtype, nan_behind=False)
    kp = c["pool"][:, 0].view(P, H, 16, D)
    kp[c["table"][0, (n - 1) // 16], :, (n - 1) % 16] = NAN
    a = run_attention(c)
    assert np.array_equal(a[:q - 1], b[:q - 1]) and np.isnan(a[q - 1, :HQ * D]).all()
    # outside the window
    c = attention_case(7, [n, n], [q, q], HQ, H, D, dtype, nan_behind=False)
    w = 40
    first = n - q - w                                     # the last position before the first query's window
    vp = c["pool"][:, 1].view(P, H, D, 16) if dtype == torch.bfloat16 else c["pool"][:, 1].view(P, H, 16, D).transpose(2, 3)
    kp = c["pool"][:, 0].view(P, H, 16, D)
    for j in range(first + 1):
        vp[c["table"][0, j // 16], :, :, j % 16] = NAN
        kp[c["table"][0, j // 16], :, j % 16] = INF
    assert np.array_equal(run_attention(c, window=w), run_attention(clean, window=w))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,q,max_kv", [(60, 1, 0), (200, 1, 0), (3000, 1, 0), (3000, 1, 600), (900, 130, 0), (3000, 130, 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_infinite_values_of_no_weight_show(D, kv, q, max_kv, dtype):
    """Key 0 scores 65536 / sqrt(D) above every other, whose weights are then exactly 0 in float32; an infinite value of one of them, in any wave's or run's share, is not lost."""
    c = attention_case(3, [kv], [q], 2, 1, D, dtype, nan_behind=False)
    P, bf = c["pool"].shape[0], dtype == torch.bfloat16
    kp = c["pool"][:, 0].view(P, 1, 16, D)
    vp = c["pool"][:, 1].view(P, 1, D, 16) if bf else c["pool"][:, 1].view(P, 1, 16, D).transpose(2, 3)
    kp.zero_()
    kp[c["table"][0, 0], :, 0, 0] = 1024
    c["q"].zero_()
    c["q"][:, ::D] = 64                                    # scores 65536 / sqrt(D) and 0
    for n, d in ((1, 3), (kv // 3, 17), (kv // 2, 40), (kv - q - 1 if q > 1 else kv - 1, 63)):
        vp[c["table"][0, n // 16], :, d, n % 16] = INF
        out = run_attention(c, max_kv=max_kv)[:q, :2 * D].reshape(q, 2, D)
        assert not np.isfinite(out[-1, :, d]).any(), (n, d)
    keep = [d for d in range(D) if d not in (3, 17, 40, 63)]
    first = c["pool"][c["table"][0, 0], 1].view(D, 16)[:, 0] if bf else c["pool"][c["table"][0, 0], 1].view(16, D)[0]
    want = np.broadcast_to(first.float().numpy()[keep], (2, len(keep)))
    assert np.array_equal(out[-1][:, keep], want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_attention_scales(scale, dtype):
    check_attention(attention_case(5, [70, 300], [3, 80], 4, 2, 64, dtype), scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_large_scores(dtype):
    """Scores in the hundreds: one key takes nearly all the weight, and the running maximum moves many times."""
    c = attention_case(9, [600, 333], [1, 200], 4, 2, 64, dtype)
    c["q"] *= 40
    check_attention(c)


@pytest.mark.parametrize("max_kv", [0, 1, 64, 5000])
def test_attention_key_hint_changes_no_result_beyond_rounding(max_kv):
    for q in (1, 90):
        check_attention(attention_case(13, [3000, 17, 900], [q, 1, q], 4, 2, 64, torch.bfloat16), max_kv=max_kv)


@pytest.mark.parametrize("n,kv_hi,q_hi,HQ,H,D", [(4096, 20, 1, 1, 1, 64), (300, 40, 3, 2, 1, 128), (100, 60, 40, 4, 2, 64),
                                                (65, 70, 30, 4, 1, 128), (64, 70, 1, 2, 2, 128)])
def test_attention_many_rows(n, kv_hi, q_hi, HQ, H, D):
    rng = np.random.default_rng(n)
    q = rng.integers(0, q_hi + 1, n)
    q[0] = q_hi
    check_attention(attention_case(n, rng.integers(0, kv_hi + 1, n), q, HQ, H, D, torch.bfloat16), causal=q_hi > 1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_starts_and_lengths_outside_their_range_are_clamped(dtype):
    c = attention_case(2, [40, 30, 50], [3, 4, 70], 4, 2, 64, dtype, nan_behind=False)
    c["row_start"] = np.array([-9, 3, 7, 2 ** 31 - 1], np.int32)
    c["kv_len"] = np.array([2 ** 31 - 1, -2 ** 31, 50], np.int32)
    c["T"] = 77
    c["table"] = np.where(c["table"] < 0, 1, c["table"]).astype(np.int32)
    q = c["q"][:77]
    want = np.zeros((77, 4, 64))
    bound = np.zeros((2, 77, 4, 64))
    bf = dtype == torch.bfloat16
    paging.attend(c["pool"].float().numpy(), bf, c["table"], c["row_start"], c["kv_len"], q.float().numpy().reshape(77, 4, 64),
                  want, bound=bound)
    got = host(serving().attend_pages(c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]),
                                      q.cuda().view(77, 4, 64)).float())
    tol = bound[0] * (2.0 ** -8 if bf else 0.0) + np.abs(want) * (2.0 ** -8 if bf else 0.0) + 1e-4 * bound[0] + 1e-30
    assert (np.abs(got - want) <= tol).all()


@pytest.fixture(params=[1100, 4096, 65536])
def wide_tables(request):
    """The same cases in tables for longer rows, which the calls are cut for: other tiles and runs of the keys."""
    global WIDTH
    WIDTH = request.param
    yield
    WIDTH = 0


@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (8, 2, 128), (7, 1, 64), (3, 3, 128), (20, 1, 128), (16, 8, 64), (8, 8, 128)])
def test_attention_in_wide_tables(wide_tables, HQ, H, D):
    for i in range(len(LENGTHS)):
        test_attention_causal(i, HQ, H, D, torch.bfloat16)
    for kv, q_len in (([50, 0, 129], [3, 9, 140]), ([1], [70]), ([700, 16], [1, 1]), ([90, 33, 64], [64, 65, 1])):
        test_attention_full(kv, q_len, HQ, H, D, torch.bfloat16)
    for w in (1, 37, 200, 100000):
        check_attention(attention_case(w, [400, 63, 700], [130, 1, 3], HQ, H, D, torch.bfloat16), window=w)


def test_attention_edges_in_wide_tables(wide_tables):
    bf = torch.bfloat16
    for q in (1, 4, 150):
        test_attention_rows_that_see_nothing(q, bf)
        test_attention_pages_outside_the_pool_are_not_seen(q, bf)
    for HQ, H, D, q in ((2, 2, 64, 4), (4, 1, 128, 4), (2, 2, 64, 150), (4, 2, 128, 200)):
        test_attention_what_is_not_seen_never_matters(HQ, H, D, q, bf)
    for scale in (0.0, -0.3, 2.0):
        test_attention_scales(scale, bf)
    test_attention_large_scores(bf)
    for D in (64, 128):
        for kv, q in ((60, 1), (3000, 1), (900, 130), (3000, 130)):
            test_attention_infinite_values_of_no_weight_show(D, kv, q, 0, bf)


@pytest.mark.parametrize("D,window", [(128, 300), (64, 450), (128, 1000)])
def test_attention_window_of_long_chunks(D, window):
    check_attention(attention_case(D, [1300, 0, 707], [600, 3, 600], 16, 8, D, torch.bfloat16), window=window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,q_len", [([300], [1]), ([300], [200]), ([2000], [33]), ([90, 300, 20], [4, 130, 1]),
                                      ([40] * 70, [1, 3] * 35)])
@pytest.mark.parametrize("front", [1, 16, 37, 130])
def test_attention_tokens_before_the_first_row(front, kv, q_len, dtype):
    c = attention_case(front, kv, q_len, 4, 2, 64, dtype)
    c["q"] = torch.cat([torch.full((front, c["q"].shape[1]), NAN, dtype=dtype), c["q"]])
    c["row_start"], c["T"] = c["row_start"] + front, c["T"] + front
    check_attention(c)                                     # (the first tokens keep what out holds, as the last do)


def test_calls_that_need_a_gradient_are_refused():
    c = attention_case(2, [40], [3], 4, 2, 64, torch.float32)
    q = c["q"][:3].cuda().view(3, 4, 64).requires_grad_()
    args = (c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), q)
    with pytest.raises(ValueError):
        serving().attend_pages(*args)
    with torch.no_grad():
        serving().attend_pages(*args)


def test_attention_is_reproducible():
    c = attention_case(17, [4000, 900, 2000], [1, 1, 1], 8, 2, 128, torch.bfloat16)
    a = run_attention(c)
    for _ in range(3):
        assert np.array_equal(run_attention(c), a)


def test_attention_long_cache_offsets():
    """A pool whose element offsets pass 2^31, read at its far end."""
    H, D, pages = 8, 128, 70000                            # 70000 * 2 * 8 * 2048 = 2.3e9 elements, 4.6 GB
    pool = torch.zeros((pages, 2, H, 16 * D), dtype=torch.bfloat16, device="cuda")
    far = torch.arange(pages - 40, pages, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    pool[far] = torch.randn((40, 2, H, 16 * D), generator=g, device="cuda").bfloat16()
    for kv, q in ((620, 1), (600, 140)):
        table = (far[torch.randperm(40, generator=g, device="cuda")]).to(torch.int32)[None].contiguous()
        x = torch.randn((q, 16, D), generator=g, device="cuda").bfloat16()
        got = serving().attend_pages(pool, table, dev([0, q]), dev([kv]), x)
        small = pool[table[0].long()].float().cpu().numpy()
        want, bound = np.zeros((q, 16, D)), np.zeros((2, q, 16, D))
        paging.attend(small, True, np.arange(40)[None], [0, q], [kv], x.float().cpu().numpy(), want, bound=bound)
        tol = bound[0] * 2.0 ** -7.9 + np.abs(want) * 2.0 ** -8 + 1e-4
        assert (np.abs(host(got.float()) - want) <= tol).all()
    # and written there
    slots = (far.to(torch.int32) * 16 + 3)
    k = torch.randn((40, H, D), generator=g, device="cuda").bfloat16()
    serving().write_pages(pool, slots, k, k)
    assert torch.equal(pool[far, 0].view(40, H, 16, D)[:, :, 3], k)
    assert torch.equal(pool[far, 1].view(40, H, D, 16)[..., 3], k)
    serving().copy_pages(pool, torch.tensor([[pages - 1, 5]], dtype=torch.int32, device="cuda"))
    assert torch.equal(pool[5], pool[pages - 1])


# ------------------------------------------------------------------- beams
def check_beams(logits, score, length, done, eos, eos_min=0, alpha=0.0):
    got = serving().select_beams(logits if torch.is_tensor(logits) else dev(logits, torch.float32), dev(score, torch.float32),
                                 dev(length), dev(done), eos, eos_min, alpha)
    lg = host(logits) if torch.is_tensor(logits) else logits
    want = paging.beams(lg, np.asarray(score, np.float32), length, done, eos, eos_min, alpha)
    for name, w in zip(("length", "done", "parent", "token"), want[1:]):
        assert np.array_equal(host(getattr(got, name)), w), (name, host(getattr(got, name)), w)
    s, w = host(got.score).astype(np.float64), want[0]
    fin = np.isfinite(w)
    assert np.array_equal(fin, np.isfinite(s)) and np.array_equal(s[~fin], w[~fin])
    # the normaliser: float32 exponentials (2^-22 relative, argument rounding 2^-24 |x - M| e^-|x - M| <= 2^-24), float64 sums
    assert (np.abs(s[fin] - w[fin]) <= 2.0 ** -21 + 2.0 ** -24 * np.abs(w[fin])).all()
    return got


@pytest.mark.parametrize("R,W,V", [(1, 1, 1), (1, 1, 2), (2, 4, 3), (1, 4, 1025), (3, 8, 1000), (5, 32, 777), (2, 5, 33000),
                                   (40, 2, 64), (1, 16, 131072), (1, 32, 20), (9, 3, 4097), (2, 32, 9000), (1, 8, 1 << 20),
                                   (2, 9, 60001)])
@pytest.mark.parametrize("alpha,eos_min", [(0.0, 0), (0.7, 12)])
def test_beam_select(R, W, V, alpha, eos_min):
    rng = np.random.default_rng(R * W + V)
    lg = (rng.standard_normal((R, W, V)) * 2.5).astype(np.float32)
    score = -np.abs(rng.standard_normal((R, W))).astype(np.float32) * 6
    length = rng.integers(0, 30, (R, W)).astype(np.int32)
    done = (rng.random((R, W)) < 0.25).astype(np.int32)
    check_beams(lg, score, length, done, V - 1, eos_min, alpha)
    # the first step: one live beam
    score[:, 1:] = -INF
    check_beams(lg, score, length * 0, done * 0, 0, eos_min, alpha)


def test_beam_select_ties_go_to_the_lowest():
    lg = np.zeros((2, 4, 300), np.float32)                 # every candidate of every beam alike
    got = check_beams(lg, np.zeros((2, 4)), np.ones((2, 4)), np.zeros((2, 4)), 299)
    assert host(got.token).tolist() == [[0, 1, 2, 3]] * 2 and host(got.parent).tolist() == [[0] * 4, [4] * 4]
    lg[:, :, [7, 255, 256]] = 3.0                          # three each
    check_beams(lg, np.zeros((2, 4)), np.ones((2, 4)), np.zeros((2, 4)), 299)
    rng = np.random.default_rng(0)
    lg = rng.integers(0, 3, (3, 8, 2000)).astype(np.float32)
    lg[1] = lg[1, :1]
    check_beams(lg, np.zeros((3, 8)), np.ones((3, 8)), np.zeros((3, 8)), 5)


def test_beam_select_odd_values():
    rng = np.random.default_rng(1)
    lg = rng.standard_normal((8, 4, 500)).astype(np.float32)
    score = -rng.random((8, 4)).astype(np.float32)
    lg[0, :, 3:] = -INF                                    # three candidates a beam
    lg[1, 0] = -INF                                        # a dead beam
    lg[2, :, 1:] = NAN
    lg[3, 1, 7] = INF                                      # no finite normaliser
    lg[4] = NAN                                            # nothing at all
    lg[5] = np.finfo(np.float32).min
    lg[6] *= 1e30
    score[6, 2] = NAN
    score[7, 1] = INF
    score[7, 2] = -INF
    done = np.zeros((8, 4), np.int32)
    done[4, 2] = done[7, 0] = 1
    check_beams(lg, score, np.full((8, 4), 3), done, 499, eos_min=5)


def test_beam_select_all_finished():
    lg = np.full((2, 3, 50), NAN, np.float32)
    got = check_beams(lg, [[-1, -3, -2], [-4, -4, -4]], np.full((2, 3), 9), np.ones((2, 3), np.int32), 20)
    assert host(got.parent).tolist() == [[0, 2, 1], [3, 4, 5]] and (host(got.length) == 9).all()


def test_beam_select_strided_logits():
    rng = np.random.default_rng(2)
    wide = dev(rng.standard_normal((3, 4, 1101)), torch.float32)
    for view in (wide[:, :, :1025], wide[:, :, 3:1028], wide[:1, :, 1:900], wide[:, :1, 5:70]):
        R, W, V = view.shape
        check_beams(view, -rng.random((R, W)).astype(np.float32), np.ones((R, W)), np.zeros((R, W)), V - 1)
    with pytest.raises(ValueError):
        serving().select_beams(wide[:, ::2].transpose(1, 2), *(dev(np.ones((3, 1101)), t) for t in
                                                             (torch.float32, torch.int32, torch.int32)), 0)


# ---------------------------------------------------------------- together
class BeamRun:
    """A beam search over a one-layer attention 'model' whose keys, values and queries are tables of the token and
    position: every step plans, copies, writes, attends, projects and selects, all on the device."""

    def __init__(self, R=3, W=4, V=120, H=2, HQ=4, D=64, m=6, dtype=torch.float32):
        g = torch.Generator().manual_seed(5)
        r = lambda *s: torch.randn(s, generator=g)
        self.R, self.W, self.V, self.n, self.m, self.eos = R, W, V, R * W, m, V - 1
        self.pages = self.n * m
        self.kt, self.vt, self.qt = r(V, H, D).to(dtype), r(V, H, D).to(dtype), r(V, HQ, D).to(dtype)
        self.pt, self.head = (r(16 * m, H, D) * 0.5).to(dtype), r(HQ * D, V) * 0.7
        self.dtype, self.H, self.HQ, self.D = dtype, H, HQ, D
        self.prompt = torch.randint(0, V - 1, (R, 19), generator=g)

    def start(self):
        """State after the prompts: one beam of each request holds the prompt, the others are dead copies of it."""
        s, n = serving(), self.n
        i32 = dict(dtype=torch.int32, device="cuda")
        self.d = {k: getattr(self, k).cuda() for k in ("kt", "vt", "qt", "pt", "head")}
        self.pools = torch.full((2, self.pages, 2, self.H, 16 * self.D), NAN, dtype=self.dtype, device="cuda")
        P = self.prompt.shape[1]
        plan = s.plan_pages(torch.zeros(n, **i32), torch.full((n,), P, **i32), torch.full((n, self.m), -1, **i32),
                            self.pages, n * P)
        tok = self.prompt.repeat_interleave(self.W, 0).reshape(-1).cuda()
        pos = plan.positions.long()
        for l in range(2):
            s.write_pages(self.pools[l], plan.slots, self.d["kt"][tok] + self.d["pt"][pos], self.d["vt"][tok])
        self.table, self.length = plan.table, plan.kv_len
        self.score = torch.tensor([[0.0] + [-INF] * (self.W - 1)] * self.R, device="cuda")
        self.gen = torch.zeros((self.R, self.W), **i32)
        self.done = torch.zeros((self.R, self.W), **i32)
        self.token = self.prompt[:, -1:].expand(-1, self.W).contiguous().to(**i32)
        self.parent = torch.arange(n, **i32)
        self.add = torch.ones(n, **i32)

    def step(self):
        """One step from the state's tensors; returns the next state's."""
        s = serving()
        plan = s.plan_pages(self.length, self.add, self.table, self.pages, self.n, parent=self.parent)
        s.copy_pages(self.pools, plan.copies)
        tok, pos = self.token.view(-1).long(), plan.positions.long()
        o = 0
        for l in range(2):
            s.write_pages(self.pools[l], plan.slots, self.d["kt"][tok] + self.d["pt"][pos], self.d["vt"][tok])
            o = o + s.attend_pages(self.pools[l], plan.table, plan.row_start, plan.kv_len, self.d["qt"][tok], max_kv=40)
        logits = (o.float().view(self.n, -1) @ self.d["head"]).view(self.R, self.W, self.V)
        b = s.select_beams(logits, self.score, self.gen, self.done, self.eos, eos_min=2, alpha=0.5)
        return plan, b

    def advance(self, plan, b):
        self.table.copy_(plan.table)
        self.length.copy_(plan.kv_len)
        self.score.copy_(b.score)
        self.gen.copy_(b.length)
        self.done.copy_(b.done)
        self.token.copy_(b.token)
        self.parent.copy_(b.parent.view(-1))

    def reference(self, steps):
        """The same search on token histories, in float64, without a cache."""
        f = lambda t: t.double()
        hist = [[self.prompt[r].tolist() for _ in range(self.W)] for r in range(self.R)]
        score = np.array([[0.0] + [-INF] * (self.W - 1)] * self.R)
        gen, done = np.zeros((self.R, self.W), np.int32), np.zeros((self.R, self.W), np.int32)
        out = []
        tok = [[h[-1] for h in row] for row in hist]
        for _ in range(steps):
            lg = np.zeros((self.R, self.W, self.V), np.float32)
            for r in range(self.R):
                for w in range(self.W):
                    ids = torch.tensor(hist[r][w] + [tok[r][w]])
                    k = f(self.kt[ids] + self.pt[torch.arange(len(ids))])
                    v, q = f(self.vt[ids]), f(self.qt[ids[-1]])
                    o = torch.cat([2 * torch.softmax(k[:, h // 2] @ q[h] / 8.0, 0) @ v[:, h // 2] for h in range(self.HQ)])
                    lg[r, w] = (o @ f(self.head)).numpy()
                    hist[r][w] = ids.tolist()
            s, n, d, p, t = paging.beams(lg, score.astype(np.float32), gen, done, self.eos, 2, 0.5)
            hist = [[list(hist[r][p[r, w] % self.W]) for w in range(self.W)] for r in range(self.R)]
            tok = t.tolist()
            score, gen, done = s, n, d
            out.append((s, n, d, p, t))
        return out


def check_run(run, got, want):
    for i, (b, (s, n, d, p, t)) in enumerate(zip(got, want)):
        assert np.array_equal(b[3], p) and np.array_equal(b[4], t) and np.array_equal(b[1], n) and np.array_equal(b[2], d), i
        fin = np.isfinite(s)
        # logits are float32 sums of 256 products of float32 attention outputs; two dozen steps of log probabilities add up
        assert (np.abs(b[0][fin] - s[fin]) <= 1e-3).all()


def test_beam_search_of_paged_sequences():
    run = BeamRun()
    run.start()
    got = []
    for _ in range(24):
        plan, b = run.step()
        assert host(plan.status).tolist() == [0, 0, 0, 0]
        run.advance(plan, b)
        got.append([host(x) for x in b])
    check_run(run, got, run.reference(24))


def test_beam_search_captured_and_replayed():
    run = BeamRun()
    want = run.reference(24)
    run.start()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        plan, b = run.step()                              # warm-up on the stream; the state does not move
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan, b = run.step()
    fresh = {k: getattr(run, k).clone() for k in ("pools", "table", "length", "score", "gen", "done", "token", "parent")}
    for rounds in range(2):                               # the whole search twice from the same graph
        for k, t in fresh.items():
            getattr(run, k).copy_(t)
        got = []
        for _ in range(24):
            graph.replay()
            run.advance(plan, b)
            got.append([host(x) for x in b])
            torch.zeros(1000, device="cuda").add_(1)      # eager work between the replays
        check_run(run, got, want)


def test_calls_on_another_stream():
    c = attention_case(21, [900, 350], [1, 70], 4, 2, 64, torch.bfloat16)
    want = run_attention(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = [run_attention(c) for _ in range(3)]
    torch.cuda.synchronize()
    for o in outs:
        assert np.array_equal(o, want)


def test_beam_select_in_place():
    """The out arrays may be the in arrays, with one launch and with two."""
    from paper_2410_13839_amd import binding as b
    rng = np.random.default_rng(8)
    for R, W, V in ((3, 4, 700), (2, 8, 20000)):
        lg, score = rng.standard_normal((R, W, V)).astype(np.float32), -rng.random((R, W)).astype(np.float32)
        ln, dn = rng.integers(1, 9, (R, W)), rng.integers(0, 2, (R, W))
        want = serving().select_beams(dev(lg, torch.float32), dev(score, torch.float32), dev(ln), dev(dn), 5, 3, 0.6)
        x = dict(score=dev(score, torch.float32), length=dev(ln), done=dev(dn), parent=dev(dn * 0), token=dev(dn * 0))
        x_lg = dev(lg, torch.float32)
        p = {k: t.data_ptr() for k, t in x.items()}
        a = b.mtp_beam_args(R, W, V, 5, 3, 0.6, x_lg.data_ptr(), V, p["score"], p["length"], p["done"], p["score"], p["length"],
                            p["done"], p["parent"], p["token"], None, 0)
        ws = torch.empty(max(1, b.mtp_beam_select_workspace_size(a)), dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        b.mtp_beam_select(a, torch.cuda.current_stream().cuda_stream)
        for k, t in x.items():
            assert np.array_equal(host(t), host(getattr(want, k))), k


class Batch:
    """One large call of every kind, whose plan, attention and selection need workspaces; inputs that can change."""

    def __init__(self, seed, n=70, m=300, H=2, HQ=8, D=128, W=8, V=30000):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.pages, self.W, self.V = n * 8 + m, W, V
        kv = rng.integers(0, 100, n)
        kv[0] = 16 * m - 40
        self.length, self.add = dev(kv), dev(rng.integers(0, 4, n))
        self.table = dev(tables(rng, kv + 4, m, self.pages))
        self.T = 4 * n
        self.pool = torch.randn((self.pages, 2, H, 16 * D), generator=g).bfloat16().cuda()
        self.k, self.v = (torch.randn((self.T, H, D), generator=g).bfloat16().cuda() for _ in range(2))
        self.q = torch.randn((self.T, HQ, D), generator=g).bfloat16().cuda()
        self.out = torch.zeros((self.T, HQ, D), dtype=torch.bfloat16, device="cuda")
        # a row alone over a long cache: its keys in runs
        self.q1, self.one = self.q[:1].clone(), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        self.logits = torch.randn((2, W, V), generator=g).cuda()
        self.score = torch.randn((2, W), generator=g).cuda()
        self.zero = torch.zeros((2, W), dtype=torch.int32, device="cuda")

    def run(self):
        s = serving()
        p = s.plan_pages(self.length, self.add, self.table, self.pages, self.T)
        s.write_pages(self.pool, p.slots, self.k, self.v)
        self.out.zero_()
        s.attend_pages(self.pool, p.table, p.row_start, p.kv_len, self.q, max_kv=5000, out=self.out)
        o1 = s.attend_pages(self.pool, p.table[:1], self.one, p.kv_len[:1], self.q1)
        b = s.select_beams(self.logits, self.score, self.zero, self.zero, 1)
        return (*p, self.out, o1, *b)


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_batches_at_once_on_two_streams():
    a, b = Batch(1), Batch(2)
    want_a, want_b = ([t.clone() for t in x.run()] for x in (a, b))
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got_a, got_b = [], []
    for _ in range(6):
        for st, x, got in ((s, a, got_a), (t, b, got_b)):
            with torch.cuda.stream(st):
                got.append([y.clone() for y in x.run()])
    torch.cuda.synchronize()
    assert all(same(g, want_a) for g in got_a) and all(same(g, want_b) for g in got_b)


def test_two_graphs_and_eager_calls_in_turn():
    """Two captured batches replayed in turn, and at once on two streams, with eager calls of a third and changed inputs
    between; every replay against the eager result of the same inputs."""
    x, y, z = Batch(3), Batch(4), Batch(5)
    want_z = [t.clone() for t in z.run()]
    graphs, outs = [], []
    for b in (x, y):
        b.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(b.run())
        graphs.append(g)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(4):
        for b in (x, y):
            b.q.mul_(-1.1)
            b.length[2:].copy_(torch.flip(b.length[2:], (0,)) // 2)
            b.logits.copy_(b.logits.roll(77, 2))
        want = [[t.clone() for t in b.run()] for b in (x, y)]
        assert same(z.run(), want_z)
        if i % 2:
            torch.cuda.synchronize()
            for st, g in zip(streams, graphs):
                with torch.cuda.stream(st):
                    g.replay()
        else:
            graphs[0].replay()
            assert same(z.run(), want_z)
            graphs[1].replay()
        torch.cuda.synchronize()
        assert same(outs[0], want[0]) and same(outs[1], want[1]), i


def test_calls_of_nothing():
    s = serving()
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")
    for n in (0, 1, 3):                                    # rows without tokens; n == 0: no rows either
        p = s.plan_pages(i(n), i(n), i(n, 700) - 1, 50, 0)
        assert host(p.row_start).tolist() == [0] * (n + 1) and host(p.status).tolist() == [0] * 4 and p.slots.shape == (0,)
        for dtype in (torch.float32, torch.bfloat16):
            pool = torch.ones((50, 2, 2, 1024), dtype=dtype, device="cuda")
            q = torch.zeros((0, 4, 64), dtype=dtype, device="cuda")
            assert s.attend_pages(pool, p.table, p.row_start, p.kv_len, q).shape == (0, 4, 64)
            s.write_pages(pool, p.slots, q[:, :2], q[:, :2])
            s.copy_pages(pool, p.copies)
            assert (pool == 1).all()
    out = torch.full((5, 4, 64), 7.0, device="cuda")       # no rows: every token keeps what out holds
    s.attend_pages(torch.ones((50, 2, 2, 1024), device="cuda"), i(0, 9), i(1), i(0), out.clone(), out=out)
    assert (out == 7.0).all()
    b = s.select_beams(torch.zeros((0, 3, 9), device="cuda"), torch.zeros((0, 3), device="cuda"), i(0, 3), i(0, 3), 1)
    assert b.token.shape == (0, 3)


def test_beam_select_most_rows():
    """The largest number of beams, of which a few requests are checked."""
    R, W, V = 2047, 32, 2049
    g = torch.Generator(device="cuda").manual_seed(4)
    lg = torch.randn((R, W, V), generator=g, device="cuda")
    score = torch.randn((R, W), generator=g, device="cuda")
    ln = torch.randint(0, 30, (R, W), generator=g, device="cuda").to(torch.int32)
    dn = (torch.rand((R, W), generator=g, device="cuda") < 0.1).to(torch.int32)
    got = serving().select_beams(lg, score, ln, dn, 2000, 5, 0.7)
    for r in (0, 1, 1023, 2046):
        want = paging.beams(*(host(t[r:r + 1]) for t in (lg, score, ln, dn)), 2000, 5, 0.7)
        for name, w in zip(("length", "done", "parent", "token"), want[1:]):
            w = w + r * W if name == "parent" else w
            assert np.array_equal(host(getattr(got, name))[r:r + 1], w), (r, name)
        assert (np.abs(host(got.score)[r:r + 1] - want[0]) <= 2.0 ** -21 + 2.0 ** -24 * np.abs(want[0])).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (6, 2, 128)])
def test_attention_many_tokens(HQ, H, D, dtype):
    """Rows of up to 90,000 tokens, a window's keys each; sampled queries against 64 bits.  Errors as in check_attention."""
    window, kv = 50, np.array([90000, 7, 31013])
    g = torch.Generator().manual_seed(HQ)
    pages = int(sum(-(-int(n) // 16) for n in kv))
    table = tables(np.random.default_rng(1), kv, 5700, pages)
    pool = torch.randn((pages, 2, H, 16 * D), generator=g).to(dtype)
    start = np.concatenate([[0], np.cumsum(kv)]).astype(np.int32)
    q = torch.randn((int(start[-1]), HQ, D), generator=g).to(dtype)
    out = host(serving().attend_pages(pool.cuda(), dev(table), dev(start), dev(kv), q.cuda(), window=window))
    bf = dtype == torch.bfloat16
    pn, qn = pool.float().numpy().astype(np.float64), q.float().numpy().astype(np.float64)
    for c, pos in ((0, 0), (0, 1), (0, 49), (0, 50), (0, 44444), (0, 89999), (1, 0), (1, 6), (2, 0), (2, 31012)):
        js = np.arange(max(0, pos - window + 1), pos + 1)
        pg = table[c, js // 16]
        k = pn[pg, 0].reshape(len(js), H, 16, D)[np.arange(len(js)), :, js % 16]
        v = pn[pg, 1].reshape((len(js), H, D, 16) if bf else (len(js), H, 16, D))
        v = (v.transpose(0, 1, 3, 2) if bf else v)[np.arange(len(js)), :, js % 16]
        for h in range(HQ):
            x, kk, vv = qn[start[c] + pos, h], k[:, h // (HQ // H)], v[:, h // (HQ // H)]
            s = kk @ x / D ** 0.5
            p = np.exp(s - s.max())
            p /= p.sum()
            mag = p @ np.abs(vv)
            ds = (D + 8) * 2.0 ** -24 * (np.abs(kk) @ np.abs(x)).max() / D ** 0.5 + 2.0 ** -22
            tol = mag * (2 * ds + 1100 * 2.0 ** -24 + (2.0 ** -8 if bf else 0.0))
            want = p @ vv
            tol = tol + np.abs(want) * (2.0 ** -8 if bf else 2.0 ** -24)
            assert (np.abs(out[start[c] + pos, h] - want) <= tol).all(), (c, pos, h)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D,kv,q_len", [(2, 2, 64, [5, 3], [9, 40]), (4, 2, 128, [30, 70], [33, 1]),
                                             (8, 8, 128, [1000, 700], [1200, 900])])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 3, 2 ** 30])
def test_attention_windows_wider_than_any_row(window, HQ, H, D, kv, q_len, dtype):
    """Such a window hides nothing, also of tiles whose first queries sit before the row's start (the last shape is the
    wide kernel's in bf16): to the bit what the call without a window gives."""
    c = attention_case(window % 1000, kv, q_len, HQ, H, D, dtype)
    if max(q_len) < 100:
        check_attention(c, window=window)
    assert np.array_equal(run_attention(c, window=window), run_attention(c))


@pytest.mark.parametrize("W,V", [(4, 9), (4, 500), (7, 7), (16, 40), (20, 2100)])
def test_beam_select_finished_beams_without_a_score(W, V):
    """A finished beam whose score is -infinity, NaN or +infinity has candidates of -infinity only, in token order like
    every other beam's of that kind; too few others are finite, so that some of them are chosen."""
    rng = np.random.default_rng(W * V)
    lg = rng.standard_normal((6, W, V)).astype(np.float32)
    lg[:, W - 1, 2:] = -INF                                # two finite candidates
    score = -rng.random((6, W)).astype(np.float32)
    done = np.ones((6, W), np.int32)
    done[:, W - 1] = 0
    for r, x in enumerate((-INF, NAN, INF)):
        score[r, :W - 1] = x                               # all of the finished
        score[3 + r, 0] = x                                # the first only
    score[3:, 1:] = -INF
    score[5] = NAN                                         # nothing at all
    for eos in (0, 3, V - 1):
        check_beams(lg, score, rng.integers(1, 9, (6, W)), done, eos, alpha=0.5)


@pytest.mark.parametrize("V", [449, 1985, 4000, 40000])
def test_beam_select_sums_exponentials_in_float64(V):
    """One logit of 0, every 64th behind it -18, the others -infinity (a lane's own logits are 64 apart): the best
    score is -log1p(n e^-18), which float32 sums around 1 would lose (e^-18 < 2^-25).  It is wrong by the exponentials'
    relative error, 2^-22 of their own and 2^-24 * 18 * log2(e) + 2^-24 * 18 of their argument, and float64 log's
    rounding of a sum near 1, 2^-52, beside the output's."""
    lg = np.full((2, 2, V), -INF, np.float32)
    lg[:, :, ::64] = -18.0
    lg[:, :, 0] = 0.0
    got = serving().select_beams(dev(lg, torch.float32), torch.zeros((2, 2), device="cuda"), dev(np.ones((2, 2))),
                                 dev(np.zeros((2, 2))), V - 2)
    n = (V + 63) // 64 - 1
    want = -np.log1p(n * np.exp(-18.0))
    s = host(got.score).astype(np.float64)
    assert (np.abs(s - want) <= -want * (2.0 ** -22 + 2.0 ** -24 * (18 * 2.45 + 1)) + 2.0 ** -52).all(), (s, want)
    assert (host(got.token) == 0).all() and host(got.parent).tolist() == [[0, 1], [2, 3]]


def test_beam_scores_that_need_a_gradient_are_refused():
    lg, score = torch.zeros((1, 2, 5), device="cuda"), torch.zeros((1, 2), device="cuda")
    i = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    for a, b in ((lg, score.clone().requires_grad_()), (lg.clone().requires_grad_(), score)):
        with pytest.raises(ValueError, match="backward"):
            serving().select_beams(a, b, i, i, 4)
        with torch.no_grad():
            assert host(serving().select_beams(a, b, i, i, 4).token).tolist() == [[0, 1]]


def test_calls_with_tangents_are_refused():
    import torch.autograd.forward_ad as fwd
    c = attention_case(2, [40], [3], 4, 2, 64, torch.float32)
    q, pool = c["q"][:3].cuda().view(3, 4, 64), c["pool"].cuda()
    where = dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"])
    k, slots = torch.zeros((3, 2, 64), device="cuda"), dev([1, 2, 3])
    lg, score = torch.zeros((1, 2, 5), device="cuda"), torch.zeros((1, 2), device="cuda")
    i = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    before = pool.clone()
    with fwd.dual_level():
        d = lambda t: fwd.make_dual(t, torch.ones_like(t))
        s = serving()
        for call in (lambda: s.attend_pages(pool, *where, d(q)), lambda: s.attend_pages(d(pool), *where, q),
                     lambda: s.attend_pages(pool, *where, q, out=d(q.clone())), lambda: s.write_pages(pool, slots, d(k), k),
                     lambda: s.write_pages(pool, slots, k, d(k)), lambda: s.copy_pages(d(pool), dev([[0, 1]])),
                     lambda: s.select_beams(d(lg), score, i, i, 4), lambda: s.select_beams(lg, d(score), i, i, 4)):
            with pytest.raises(ValueError, match="forward-mode"):
                call()
        assert torch.equal(pool.view(torch.int32), before.view(torch.int32))   # (NaN behind the keys)
        s.attend_pages(pool, *where, q)                    # (plain tensors inside dual_level)


def test_calls_inside_a_trace_are_refused():
    c = attention_case(2, [40], [3], 4, 2, 64, torch.float32)
    q = c["q"][:3].cuda().view(3, 4, 64)
    args = c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"])
    with pytest.raises(ValueError, match="traced"):
        torch.jit.trace(lambda x: serving().attend_pages(*args, x), (q,))
    assert torch.isfinite(serving().attend_pages(*args, q)).all()


def test_what_calls_write_counts_as_changed():
    """The written tensors' versions move on, views of them and inference tensors included, so that a backward pass that
    saved one says so; what a call only reads keeps its version."""
    s = serving()
    pools = torch.zeros((2, 9, 2, 2, 1024), device="cuda")
    x = torch.ones(1, device="cuda", requires_grad=True)
    k, slots, q = torch.ones((3, 2, 64), device="cuda"), dev([1, 2, 3]), torch.ones((3, 4, 64), device="cuda")
    table, start, kv = dev([[0, 1]]), dev([0, 3]), dev([20])
    buf = torch.zeros((5, 4, 64), device="cuda")
    length = dev([3])
    calls = {"write": (pools, lambda: s.write_pages(pools[1], slots, k, k)),
             "copy": (pools, lambda: s.copy_pages(pools, dev([[0, 1]]))),
             "attend": (buf, lambda: s.attend_pages(pools[0], table, start, kv, q, out=buf[1:4])),
             "plan": (table, lambda: s.plan_pages(length, dev([1]), table, 9, 2, out_table=table))}
    reads = (k, slots, q, start, kv, length)
    for name, (t, call) in calls.items():
        old, olds = t._version, [r._version for r in reads]
        saved = (x * t.float()).sum() if t.dtype == torch.float32 else None
        call()
        assert t._version > old and [r._version for r in reads] == olds, name
        if saved is not None:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                saved.backward()
    with torch.inference_mode():
        p = torch.zeros((9, 2, 2, 1024), device="cuda")
        s.write_pages(p, slots, k, k)
        assert float(p.sum()) == 3 * 2 * 2 * 64
        s.attend_pages(p, table, start, kv, q, out=torch.empty_like(q))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [0.0, -0.0, 0.125, -0.125])
@pytest.mark.parametrize("HQ,H,D,q", [(2, 2, 64, 3), (8, 8, 128, 900)])
def test_attention_queries_that_are_not_numbers(HQ, H, D, q, scale, dtype):
    """A query that holds a NaN or an infinity (0 x infinity included, so also with scale 0) gets NaN in that head, its
    neighbours what they get without it; the second shape is the wide kernel's in bf16."""
    c = attention_case(11, [1000], [q], HQ, H, D, dtype)
    want = run_attention(c, scale=scale)[:q].reshape(q, HQ, D)
    assert np.isfinite(want).all()
    hit = np.zeros((q, HQ), bool)
    x = c["q"][:q].view(q, HQ, D)
    for i, (t, h, d, value) in enumerate([(0, 0, 5, NAN), (1, 1, D - 1, NAN), (2, 0, 9, INF), (q - 1, HQ - 1, 0, -INF)]):
        x[t, h, d] = value
        hit[t, h] = True
    got = run_attention(c, scale=scale)[:q].reshape(q, HQ, D)
    if scale == 0:
        assert np.isnan(got[hit]).all()
    else:                                                  # (infinite scores: NaN, or none but -infinite ones: zeros)
        assert np.isnan(got[hit][[0, 1]]).all()
    assert np.array_equal(got[~hit], want[~hit])


@pytest.mark.parametrize("W,V", [(3, 5), (4, 300), (7, 2500), (16, 400), (32, 9000)])
def test_beam_select_scores_that_rounding_makes_equal(W, V):
    """Scores of -1e30 swallow the log probabilities in float64: a beam's own candidates still go by their logits."""
    rng = np.random.default_rng(W + V)
    lg = (rng.standard_normal((3, W, V)) * 2).astype(np.float32)
    lg[1] = np.round(lg[1])                                # and many equal logits
    score = np.full((3, W), -1e30, np.float32)
    score[2] = -np.float32(1e30) * rng.integers(1, 3, W).astype(np.float32)
    got = check_beams(lg, score, np.ones((3, W)), np.zeros((3, W)), V - 1)
    for r in range(2):
        assert (host(got.parent)[r] == r * W).all()
        assert host(got.token)[r].tolist() == np.lexsort((np.arange(V), -lg[r, 0]))[:W].tolist()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,q_len,max_kv", [([40, 300], [1, 3], 0), ([2000, 700], [1, 1], 0), ([1500, 900], [140, 200], 0),
                                             ([3000], [130], 600)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_scores_of_infinity(D, kv, q_len, max_kv, dtype):
    """Keys of -infinity in a dimension where the queries are positive score -infinity, those of +infinity infinity.
    All keys of the first row but the last few score -infinity: they have no weight.  Then all of its first head do:
    zeros; and one of its second head scores infinity: NaN."""
    c = attention_case(5, kv, q_len, 2, 2, D, dtype, nan_behind=False)
    pages, T = c["pool"].shape[0], c["T"]
    kp = c["pool"][:, 0].view(pages, 2, 16, D)
    x = c["q"][:T].view(T, 2, D)
    x[:, :, 0] = x[:, :, 0].abs() + 0.1                    # dimension 0: positive
    low = kv[0] - q_len[0] - 2                             # positions of the first row that score -infinity, in both heads
    for j in range(low):
        kp[c["table"][0, j // 16], :, j % 16, 0] = -INF
    tame = c["pool"].clone()
    tame[:, 0] = torch.where(torch.isinf(tame[:, 0]), 0.0, tame[:, 0].float()).to(dtype)
    qn = c["q"].float().numpy()[:, :2 * D].reshape(-1, 2, D)
    args = (dtype == torch.bfloat16, c["table"], c["row_start"], c["kv_len"], qn[:T])
    want, bound, unused = np.zeros((T, 2, D)), np.zeros((2, T, 2, D)), np.zeros((2, T, 2, D))
    with np.errstate(invalid="ignore"):
        paging.attend(c["pool"].float().numpy(), *args, want, bound=unused)
        paging.attend(tame.float().numpy(), *args, np.zeros((T, 2, D)), bound=bound)
    # (check_attention's tolerance, the scores' error from the finite keys)
    u = 2.0 ** -24
    bf = dtype == torch.bfloat16
    ds = (D + 8) * u * bound[1] + 4 * u
    tol = unused[0] * (2 * ds + 1100 * u + (2.0 ** -8 if bf else 0.0)) + np.abs(want) * (2.0 ** -8 if bf else u) + 1e-30
    got = run_attention(c, max_kv=max_kv)[:T].reshape(T, 2, D)
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all()
    for j in range(low, kv[0]):
        kp[c["table"][0, j // 16], 0, j % 16, 0] = -INF
    kp[c["table"][0, 3 // 16], 1, 3, 0] = INF
    got = run_attention(c, max_kv=max_kv)[:T].reshape(T, 2, D)
    assert (got[:q_len[0], 0] == 0).all() and np.isnan(got[:q_len[0], 1]).all()
    assert np.isfinite(got[q_len[0]:]).all()


@pytest.mark.parametrize("kv,q_len,HQ,H,D,dtype,window", [
    ([32768], [128], 1, 1, 128, torch.bfloat16, 0), ([65536], [128], 1, 1, 64, torch.bfloat16, 0),
    ([40000, 17000, 300], [90, 100, 40], 2, 1, 128, torch.bfloat16, 0), ([131072], [1], 1, 1, 64, torch.bfloat16, 0),
    ([90000, 70000, 20], [2, 1, 1], 4, 1, 64, torch.float32, 0), ([80000], [3], 1, 1, 128, torch.float32, 70001),
    ([66000], [2], 8, 1, 128, torch.bfloat16, 0)])
def test_attention_many_runs(kv, q_len, HQ, H, D, dtype, window):
    """Rows of more than 64 runs, which a lane of a join takes several of (up to 256 runs, the second shape)."""
    check_attention(attention_case(sum(kv) % 97, kv, q_len, HQ, H, D, dtype), window=window)
