"""Attention that adds up the cached tokens' weights, on the GPU against a plain
implementation in 64 bits (oracle/speculative.py)."""
import numpy as np
import pytest

from oracle import speculative

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


def case(seed, kv, q_len, HQ, H, D, dtype, wide=0, front=0):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    kv, q_len = np.asarray(kv), np.asarray(q_len)
    need = [-(-int(n) // 16) for n in kv]
    m, pages = max(1, max(need)) + seed % 3 + wide, sum(need) + 3
    order, at = rng.permutation(pages), 0
    table = np.full((len(kv), m), -1, np.int32)
    for c, k in enumerate(need):
        table[c, :k] = order[at:at + k]
        at += k
    pool = torch.randn((pages, 2, H, 16 * D), generator=g).to(dtype)
    kp = pool[:, 0].view(pages, H, 16, D)
    for c, n in enumerate(kv):                   # what lies behind a row's last key must not matter
        if n % 16:
            kp[table[c, n // 16], :, n % 16:] = NAN if c % 2 else INF
            pool[table[c, n // 16], 1] = 0.0
    T = int(q_len.sum()) + front
    q = (torch.randn((T, HQ, D), generator=g) * 1.5).to(dtype)
    start = (front + np.concatenate([[0], np.cumsum(q_len)])).astype(np.int32)
    weights = (rng.random((len(kv), H, 16 * m + seed % 2)) * 3).astype(np.float32)
    weights[:, :, -1] = NAN                      # nobody's, where the table is wider than the rows
    return dict(pool=pool, table=table, row_start=start, kv_len=kv.astype(np.int32), q=q, weights=weights)


def check(c, causal=True, window=0, scale=None, max_kv=0, copies=1):
    """A probability is a score's exponential times a factor: the score, a float32 sum of D products and a scaling, is within
    (D + 8) 2^-24 of the sum of their magnitudes, the reference likewise, the exponential's argument and value within 8 x
    2^-24, the factor's sum of at most 64 partial roundings a merge within 1100 x 2^-24 (as for the attention's output); the
    sum over the queries rounds once a term, and once more for what was there.  copies: rows like the one that c has."""
    bf = c["pool"].dtype == torch.bfloat16
    D = c["q"].shape[2]
    want = c["weights"].astype(np.float64)
    pool = c["pool"].float().numpy()
    off, count = speculative.attention_weights(pool, bf, c["table"], c["row_start"], c["kv_len"], c["q"].float().numpy(), want,
                                               causal, window, scale)
    if copies > 1:
        n = int(c["row_start"][1])
        c = dict(c, table=np.repeat(c["table"], copies, 0), kv_len=np.repeat(c["kv_len"], copies), q=c["q"].repeat(copies, 1, 1),
                 row_start=np.arange(copies + 1, dtype=np.int32) * n, weights=np.repeat(c["weights"], copies, 0))
        want, off, count = (np.repeat(x, copies, 0) for x in (want, off, count))
    u = 2.0 ** -24
    args = (c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), c["q"].cuda())
    kw = dict(causal=causal, window=window, scale=scale, max_kv=max_kv)
    w = dev(c["weights"], torch.float32)
    before = w._version
    out = serving().attend_pages(*args, **kw, weights=w)
    assert w._version > before
    alone = serving().attend_pages(*args, **kw)
    live = slice(int(c["row_start"][0]), int(c["row_start"][-1]))
    assert torch.equal(out[live].view(torch.int16 if bf else torch.int32), alone[live].view(torch.int16 if bf else torch.int32))
    got = w.cpu().numpy()
    worst = 0.0
    for r, n in enumerate(c["kv_len"]):
        n = min(max(int(n), 0), 16 * c["table"].shape[1])
        assert np.array_equal(got[r, :, n:], c["weights"][r, :, n:], equal_nan=True)           # behind the row's keys
        g, x = got[r, :, :n], want[r, :, :n]
        added = x - np.where(count[r, :, :n] > 0, 0.0, x)
        tol = 2 * (D + 8) * u * off[r, :, :n] + (1120 + count[r, :, :n]) * u * added + 2 * u * np.abs(x) + 1e-30
        err = np.abs(g - x) / tol
        if err.size:
            worst = max(worst, err.max())
        assert not err.size or err.max() <= 1.0, (r, err.max())
    again = dev(c["weights"], torch.float32)
    serving().attend_pages(*args, **kw, weights=again)
    assert torch.equal(again.view(torch.int32), w.view(torch.int32))                           # the same sums, bit for bit
    return worst


LENGTHS = [
    ([1], [1]), ([16], [1]), ([17], [4]), ([33], [33]), ([5, 1, 64], [5, 1, 3]),
    ([100, 0, 31, 48, 7], [1, 0, 31, 2, 7]), ([1075], [4]), ([65, 129, 200], [65, 70, 16]),
    ([513, 40, 1, 777], [1, 1, 1, 1]), ([300, 301], [257, 130]), ([40, 20], [50, 21]), ([2100], [1]),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (8, 2, 128), (7, 1, 64), (3, 3, 128), (20, 1, 128), (40, 2, 64)])
@pytest.mark.parametrize("i", range(len(LENGTHS)))
def test_weights_causal(i, HQ, H, D, dtype):
    kv, q_len = LENGTHS[i]
    check(case(i + 10 * HQ + D, kv, q_len, HQ, H, D, dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (12, 4, 128), (16, 1, 64)])
@pytest.mark.parametrize("kv,q_len", [([50, 0, 129], [3, 9, 140]), ([1], [70]), ([700, 16], [1, 1]), ([90, 33, 64], [64, 65, 1])])
def test_weights_full(kv, q_len, HQ, H, D, dtype):
    check(case(len(kv) + HQ, kv, q_len, HQ, H, D, dtype), causal=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window", [1, 2, 16, 37, 200, 100000, 2 ** 31 - 1])
def test_weights_window(window, dtype):
    check(case(window % 1000, [400, 63, 700], [130, 1, 3], 4, 2, 64, dtype), window=window)


@pytest.mark.parametrize("HQ,H,D,kv,q_len", [(8, 2, 128, [600, 300], [300, 40]), (4, 4, 64, [900, 500, 130], [500, 120, 130]),
                                             (16, 2, 64, [700], [260]), (6, 2, 128, [1500, 64], [200, 64])])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 150), (False, 0)])
def test_weights_chunks(HQ, H, D, kv, q_len, causal, window):
    check(case(HQ + D, kv, q_len, HQ, H, D, torch.bfloat16), causal, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
@pytest.mark.parametrize("q", [2, 150])
def test_weights_scales(q, scale, dtype):
    check(case(3, [300, 200], [q, 1], 8, 2, 64, dtype), scale=scale)


@pytest.mark.parametrize("max_kv", [0, 1, 300, 5000])
@pytest.mark.parametrize("q", [1, 90])
def test_weights_key_hint(q, max_kv):
    check(case(5, [3000, 40], [q, 1], 4, 2, 64, torch.bfloat16, wide=60), max_kv=max_kv)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q", [1, 4, 140])
def test_weights_pages_outside_the_pool(q, dtype):
    c = case(7, [200, 180], [q, q], 4, 2, 64, dtype)
    c["table"][0, 0], c["table"][0, 3], c["table"][1, 5] = -1, c["pool"].shape[0], 2 ** 31 - 1
    check(c)
    check(c, causal=False)
    c["table"][0] = -1                           # a row that sees nothing
    check(c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q", [1, 3, 130])
def test_weights_of_queries_and_keys_that_are_not_numbers(q, dtype):
    c = case(8, [250, 140], [q, q], 4, 2, 64, dtype)
    c["q"][0, 1], c["q"][min(1, 2 * q - 1), 2, 3] = NAN, INF
    check(c)
    kp = c["pool"][:, 0].view(-1, 2, 16, 64)
    kp[c["table"][0, 2], 0, 5] = NAN             # every query of the row that sees it comes to nothing
    kp[c["table"][1, 4], 1, 7, 0] = INF
    check(c)
    check(c, window=20)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights_tokens_before_the_first_row_and_clamped_lengths(dtype):
    check(case(9, [60, 40], [3, 30], 4, 2, 64, dtype, front=5))
    c = case(10, [60, 40], [3, 30], 4, 2, 64, dtype)
    c["kv_len"] = np.array([2 ** 31 - 1, -3], np.int32)
    c["table"][0] = np.arange(c["table"].shape[1]) % c["pool"].shape[0]
    c["pool"] = torch.randn(c["pool"].shape, generator=torch.Generator().manual_seed(1)).to(dtype)
    check(c)


def test_weights_of_shared_pages_are_each_row_s_own():
    """Rows of one table entry (beams) have sums of their own."""
    c = case(11, [100, 100, 100], [1, 1, 1], 4, 2, 64, torch.bfloat16)
    c["table"][1], c["table"][2] = c["table"][0], c["table"][0]
    check(c)


def test_weights_many_rows():
    rng = np.random.default_rng(2)
    check(case(12, rng.integers(1, 40, 300), rng.integers(0, 2, 300), 2, 1, 64, torch.bfloat16))


@pytest.mark.parametrize("HQ,H,D,kv,q,copies,dtype,window", [
    (128, 128, 64, 1100, 1, 40, torch.bfloat16, 0),      # one workgroup takes both blocks of a row and head: scores stored,
    (128, 128, 64, 300, 12, 64, torch.bfloat16, 0),      # formed again,
    (128, 128, 64, 300, 18, 64, torch.float32, 40),
    (512, 128, 64, 300, 18, 64, torch.bfloat16, 0),      # and in the tiles of many query rows
    (512, 128, 64, 420, 18, 64, torch.bfloat16, 40)])
def test_weights_of_more_rows_and_heads_than_workgroups(HQ, H, D, kv, q, copies, dtype, window):
    check(case(15, [kv], [q], HQ, H, D, dtype), window=window, copies=copies)


@pytest.mark.parametrize("q", [1, 12, 140])
def test_weights_in_a_pool_past_32_bits(q):
    """Pages beyond 2^31 elements and 2^32 bytes give what they give in a small pool."""
    c = case(16, [333, 190], [q, q], 16, 8, 128, torch.bfloat16)
    small = c["pool"].cuda()
    n, far = small.shape[0], 70000
    big = torch.empty((far, *small.shape[1:]), dtype=torch.bfloat16, device="cuda")
    big[far - n:] = small
    assert big.numel() > 2 ** 31
    res = []
    for pool, base in ((small, 0), (big, far - n)):
        w = dev(c["weights"], torch.float32)
        t = np.where(c["table"] < 0, -1, c["table"] + base)
        out = serving().attend_pages(pool, dev(t), dev(c["row_start"]), dev(c["kv_len"]), c["q"].cuda(), weights=w)
        res.append((out.view(torch.int16), w.view(torch.int32)))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_weights_of_nothing():
    c = case(13, [20, 30], [0, 0], 2, 1, 64, torch.bfloat16)
    c["q"] = c["q"][:0]
    w = dev(c["weights"], torch.float32)
    s = serving()
    s.attend_pages(c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), c["q"].cuda(), weights=w)
    assert np.array_equal(w.cpu().numpy(), c["weights"], equal_nan=True)


def test_weights_refuses():
    c = case(14, [20, 30], [1, 1], 4, 2, 64, torch.bfloat16)
    w = dev(c["weights"], torch.float32)
    args = (c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), c["q"].cuda())
    for bad in (w.double(), w[:1], w[:, :1], w[..., :16 * c["table"].shape[1] - 1].contiguous(), w.transpose(0, 1), w.cpu(), w[0],
                w.clone().requires_grad_()):
        with pytest.raises(ValueError):
            serving().attend_pages(*args, weights=bad)


@pytest.mark.parametrize("HQ,H,D,kv,q_len", [
    (32, 8, 128, [500, 260, 130, 700], [130, 129, 130, 1]),      # whole
    (32, 8, 128, [1030], [70]), (12, 4, 128, [900, 2000], [65, 130]),                # up to four runs of keys, joined
    (16, 4, 128, [4100], [64]), (36, 2, 128, [3000, 2900], [50, 33]),                # more of them; two blocks of heads
    (32, 8, 128, [1500, 1000, 40], [9, 8, 10]),                  # few queries a row
    (8, 8, 64, [1030], [1000]), (8, 8, 64, [4000], [257])])
def test_weights_many_queries(HQ, H, D, kv, q_len):
    """Enough work for the attention's kernel for many query rows: heads of 128, and runs of keys in several workgroups."""
    check(case(3 * (HQ + D), kv, q_len, HQ, H, D, torch.bfloat16))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kw", [dict(causal=False), dict(window=950), dict(scale=0.0), dict(scale=-0.2), dict(scale=0.0, causal=False)])
def test_weights_many_queries_of_every_form(D, kw):
    c = case(6, [1100, 600], [75, 65], 64, 8, D, torch.bfloat16)
    check(c, **kw)
    c["table"][0, 3], c["table"][0, 60], c["table"][1, 5] = -1, c["pool"].shape[0], -2 ** 31
    c["q"][5, 1] = NAN
    check(c, **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("HQ,H,D", [(2, 2, 64), (2, 1, 128)])
@pytest.mark.parametrize("q", [1, 60])
def test_weights_of_few_runs(q, HQ, H, D, dtype):
    """Two to four runs of keys, whose sums go along with the joins or follow them."""
    check(case(0, [528], [q], HQ, H, D, dtype))


# (the kernels that form scores again, and the attention's that they go with: the same products in the same order)
@pytest.mark.parametrize("HQ,H,D,kv,q,dtype", [
    (4, 2, 64, 300, 3, torch.bfloat16), (4, 2, 128, 600, 1, torch.float32),          # stored
    (4, 2, 64, 300, 20, torch.bfloat16), (4, 2, 64, 300, 30, torch.float32), (8, 2, 128, 300, 40, torch.float32),
    (64, 8, 128, 1100, 75, torch.bfloat16), (64, 8, 64, 1100, 130, torch.bfloat16)])  # many query rows
@pytest.mark.parametrize("scale", [0.125, -0.125])
def test_weights_of_large_scores(HQ, H, D, kv, q, dtype, scale):
    """Each query is a key of its own times +-1: its score, 10^8, lies so far above the others that the key gets the whole
    weight, however the score rounds (steps of 8 at 1.4 x 10^8).  Few query rows: the reference is the key's own score, the
    weight 1 exactly.  Many: the reference is off by a rounding, the weight e times 1 / e of some e: the quotient's rounding
    and the product's, 2^-24 each, and one a sum."""
    c = case(0, [kv], [q], HQ, H, D, dtype)
    keys = (torch.randn((kv, H, D), generator=torch.Generator().manual_seed(1)) * (3000.0 if D == 64 else 2100.0)).to(dtype)
    at = torch.arange(kv)
    c["pool"][:, 0].view(-1, H, 16, D)[torch.tensor(c["table"][0]).long()[at // 16], :, at % 16] = keys
    rng = np.random.default_rng(2)
    want = np.zeros((H, kv))
    for i in range(q):
        for h in range(HQ):
            j = int(rng.integers(0, kv - q + i + 1))
            c["q"][i, h] = keys[j, h // (HQ // H)] * (1 if scale > 0 else -1)
            want[h // (HQ // H), j] += 1.0
    k = keys.double()
    s = torch.einsum("jhd,ihd->hij", k, k) * 0.125
    gap = torch.diagonal(s, dim1=1, dim2=2)[:, :, None] - s
    assert (gap + torch.eye(kv).double() * 1e9).min() > 1e6
    w = torch.zeros(c["weights"].shape, device="cuda")
    serving().attend_pages(c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), c["q"].cuda(), scale=scale,
                           weights=w)
    assert (np.abs(w.cpu().numpy()[0, :, :kv] - want) <= want * (2 + want) * (2.0 ** -24 if HQ == 64 else 0.0)).all()


@pytest.mark.parametrize("q,D,rows", [(75, 128, 2), (75, 64, 2), (7, 128, 10)])
def test_weights_of_scale_0_where_products_overflow(q, D, rows):
    """Scores of scale 0 are 0, though a product would be infinite: out is the mean of the values, the weights are even.
    (1 over the keys seen, rounded to float32 twice at most, and a rounding a sum)."""
    c = case(0, [1100] * rows, [q] * rows, 64, 8, D, torch.bfloat16)
    c["q"] *= 1e20
    c["pool"][:, 0] *= 1e20
    w = torch.zeros(c["weights"].shape, device="cuda")
    out = serving().attend_pages(c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]), c["q"].cuda(), scale=0.0,
                                 weights=w)
    assert torch.isfinite(out).all()
    seen = np.arange(1100 - q, 1100)[:, None] + 1
    want = 8 * ((np.arange(1100)[None] < seen) / seen).sum(0)
    assert (np.abs(w.cpu().numpy()[:, :, :1100] - want) <= want * (8 * q + 1104) * 2.0 ** -24).all()


@pytest.mark.parametrize("HQ,H,D,kv,q,dtype", [(8, 2, 64, [300, 90], 2, torch.bfloat16), (8, 2, 64, [300, 90], 20, torch.bfloat16),
                                               (8, 2, 128, [300, 90], 30, torch.float32), (5, 1, 64, [200, 150], 70, torch.bfloat16),
                                               (32, 8, 128, [900, 400], 90, torch.bfloat16)])
def test_weights_of_queries_within_a_wider_buffer(HQ, H, D, kv, q, dtype):
    """Queries from one QKV buffer, an output beside others: the bits of tight ones, and what lies around stays."""
    c = case(3, kv, [q] * len(kv), HQ, H, D, dtype)
    args = (c["pool"].cuda(), dev(c["table"]), dev(c["row_start"]), dev(c["kv_len"]))
    T = c["q"].shape[0]
    w = dev(c["weights"], torch.float32)
    out = serving().attend_pages(*args, c["q"].cuda(), weights=w)
    wide = torch.full((T, (HQ + 2 * H) * D), 3.0, dtype=dtype, device="cuda")
    wide[:, :HQ * D] = c["q"].cuda().view(T, -1)
    room = torch.full((T + 1, HQ * D + 16), 7.0, dtype=dtype, device="cuda")
    w2 = dev(c["weights"], torch.float32)
    serving().attend_pages(*args, wide[:, :HQ * D].view(T, HQ, D), weights=w2, out=room[:T, 8:8 + HQ * D].view(T, HQ, D))
    assert torch.equal(w.view(torch.int32), w2.view(torch.int32))
    assert torch.equal(room[:T, 8:8 + HQ * D].reshape(T, HQ, D), out)
    assert (room[T:] == 7).all() and (room[:, :8] == 7).all() and (room[:, 8 + HQ * D:] == 7).all() and (wide[:, HQ * D:] == 3).all()
