"""The operators of speculative serving without a GPU: the library's refusals
(every one before any launch), the argument structs' layout, and pins of the
oracle."""
import math

import numpy as np
import pytest

from oracle import speculative

INF, NAN = float("inf"), float("nan")


def _b():
    from paper_2410_13839_amd import binding
    return binding


def _with(a, kw):
    for k, v in kw.items():
        at, name = a, k
        if "." in k:
            inner, name = k.rsplit(".", 1)
            for part in inner.split("."):
                at = getattr(at, part)
        setattr(at, name, v)
    return a


def _cache():
    b = _b()
    return b.mtp_cache(4096, b.MTP_DTYPE_BF16, 10, 4, 64)


def _refused(call, args, code=None):
    b = _b()
    with pytest.raises(b.MTPError) as e:
        call(args, 0)
    assert e.value.code == (b.MTP_EINVAL if code is None else code)


# ----------------------------------------------------------------- rotary
BAD_ROTARY = [dict(freq=0), dict(freq=260), dict(pairs=0), dict(pairs=33), dict(layout=2), dict(layout=-1), dict(inverse=2),
              dict(magnitude=NAN), dict(magnitude=INF)]


def _rotary():
    return _b().mtp_rotary(256, 32, 0, 0, 1.0)


def _rotate(kw):
    b = _b()
    return _with(b.mtp_rotate_args(_rotary(), b.MTP_DTYPE_BF16, 5, 2, 64, 256, 1024, 2048, 128, 128), kw)


def _write_rotated(kw):
    b = _b()
    write = b.mtp_write_args(_cache(), 5, 256, 512, 1024, 256, 256)
    return _with(b.mtp_write_rotated_args(write, _rotary(), 256, 8, 1024, 2048, 512, 512), kw)


@pytest.mark.parametrize("kw", [{"rotary." + k: v for k, v in kw.items()} for kw in BAD_ROTARY] +
                         [dict(dtype=2), dict(n_tokens=-1), dict(n_heads=0), dict(n_heads=1025), dict(head_dim=4),
                          dict(head_dim=68), dict(head_dim=1032, x_stride=4096, out_stride=4096),
                          dict(n_tokens=1 << 30, n_heads=2), dict(positions=0), dict(positions=258), dict(x=0), dict(x=1032),
                          dict(out=0), dict(out=2056), dict(x_stride=120), dict(x_stride=132), dict(out_stride=127)])
def test_rotate_refuses(kw):
    _refused(_b().mtp_rotate, _rotate(kw))


@pytest.mark.parametrize("kw", [{"rotary." + k: v for k, v in kw.items()} for kw in BAD_ROTARY] +
                         [{"write.cache.pool": 0}, {"write.cache.head_dim": 96}, {"write.n_tokens": -1}, {"write.slots": 0},
                          {"write.slots": 258}, {"write.k": 0}, {"write.v": 520}, {"write.k_stride": 255},
                          {"write.v_stride": 248}, dict(positions=0), dict(n_heads=0), dict(n_heads=1025), dict(q=0),
                          dict(q=1032), dict(out=0), dict(q_stride=504), dict(out_stride=516)])
def test_write_rotated_refuses(kw):
    _refused(_b().mtp_pages_write_rotated, _write_rotated(kw))


def test_rotary_calls_of_nothing():
    b = _b()
    b.mtp_rotate(_rotate(dict(n_tokens=0, x=0, out=0, positions=0)), 0)
    b.mtp_pages_write_rotated(_write_rotated({"write.n_tokens": 0, "q": 0}), 0)
    for call in (b.mtp_rotate, b.mtp_pages_write_rotated):
        _refused(call, None)


def test_oracle_rotation_is_a_complex_product():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 2, 16))
    pos, freq = np.array([0, 7, -1, 90000]), 100.0 ** (-np.arange(5) / 5)
    for neighbours in (False, True):
        y = speculative.rotate(x, pos, freq, neighbours, 1.5)
        a, b = (slice(0, 10, 2), slice(1, 10, 2)) if neighbours else (slice(0, 5), slice(5, 10))
        z = (x[..., a] + 1j * x[..., b]) * 1.5 * np.exp(1j * pos[:, None] * freq)[:, None]
        live = pos >= 0
        assert np.allclose(y[live][..., a], z.real[live]) and np.allclose(y[live][..., b], z.imag[live])
        assert np.array_equal(y[..., 10:], x[..., 10:]) and np.array_equal(y[~live], x[~live])
        back = speculative.rotate(y, pos, freq, neighbours, 1 / 1.5, inverse=True)
        assert np.allclose(back, x)


# ----------------------------------------------------------- verification
def _verify(kw):
    b = _b()
    return _with(b.mtp_verify_args(3, 40, 90000, 16, 89999, 5, 0.7, 256, 512, 90000, 90000, 768, 1024, 1280, 1536, 2048, 2304,
                                   2560, 2816, 3328, 4096, 1 << 20), kw)


@pytest.mark.parametrize("kw", [dict(n_rows=-1), dict(n_rows=4097), dict(n_tokens=-1), dict(n_tokens=1 << 24), dict(vocab=0),
                                dict(vocab=1 << 24), dict(width=0), dict(width=257), dict(eos_id=-2), dict(eos_id=90000),
                                dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=INF), dict(temperature=1e-310),
                                dict(n_rows=4096, width=256), dict(logits=0), dict(logits=258), dict(draft=514), dict(ld=89999),
                                dict(draft_ld=89999), dict(tokens=0), dict(row_start=0), dict(row_start=1026), dict(uniforms=0),
                                dict(len=0), dict(token=0), dict(prob=0), dict(count=0), dict(accepted=0), dict(done=0),
                                dict(workspace=0), dict(workspace=4096 + 128)])
def test_verify_refuses(kw):
    _refused(_b().mtp_verify_drafts, _verify(kw))


def test_verify_workspace():
    b = _b()
    need = b.mtp_verify_drafts_workspace_size(_verify({}))
    assert 0 < need <= 1 << 20
    _refused(b.mtp_verify_drafts, _verify(dict(workspace_bytes=need - 1)), b.MTP_ENOMEM)
    assert b.mtp_verify_drafts_workspace_size(_verify(dict(vocab=1000, width=4, eos_id=-1))) == 0
    with pytest.raises(b.MTPError):
        b.mtp_verify_drafts_workspace_size(_verify(dict(vocab=0)))
    b.mtp_verify_drafts(_verify(dict(n_rows=0, logits=0, token=0)), 0)
    _refused(b.mtp_verify_drafts, None)


def test_oracle_verification_of_a_hand_example():
    p = np.array([[0.5, 0.3, 0.2], [0.1, 0.1, 0.8], [0.25, 0.5, 0.25]])
    q = np.array([[0.2, 0.6, 0.2], [0.1, 0.1, 0.8], [1.0, 1.0, 1.0]])
    run = lambda u, draft=np.log(q), **kw: speculative.verify(np.log(p), [7, 1, 2], [0, 3], u, 3, draft, **kw)
    # 0.6 u < 0.3 passes; 0.8 u < 0.8 always; then 0.25 | 0.75 | 1
    r = run([0.7, 0.49, 0.9])
    assert r["token"].tolist() == [[1, 2, 1]] and r["accepted"].tolist() == [2] and r["count"].tolist() == [3]
    assert np.allclose(r["prob"], [[0.3, 0.8, 0.5]])
    # refused: what is left of p - q is all at 0
    r = run([0.99, 0.51, 0.0])
    assert r["token"].tolist() == [[0, -1, -1]] and r["accepted"].tolist() == [0]
    # certain drafts: u < p; what is left has the refused one taken out, 0.5 | 0.7
    assert run([0.72, 0.3, 0.0], None)["token"].tolist() == [[2, -1, -1]]
    assert run([0.71, 0.3, 0.0], None)["token"].tolist() == [[0, -1, -1]]
    assert run([0.0, 0.29, 0.79], None)["accepted"].tolist() == [2]
    # an end among the accepted: nothing behind it; masked, it is refused
    r = run([0.0, 0.0, 0.0], eos_id=1)
    assert r["token"].tolist() == [[1, -1, -1]] and r["done"].tolist() == [1] and r["accepted"].tolist() == [2]
    r = run([0.0, 0.0, 0.0], eos_id=1, eos_min=4, length=[3])
    assert r["token"].tolist() == [[0, -1, -1]] and r["done"].tolist() == [0]
    assert run([0.9, 0.9, 0.9], temperature=0)["token"].tolist() == [[0, -1, -1]]


def test_oracle_verification_gives_the_target_distribution():
    """Over a grid of both uniforms and the drafts' own probabilities, the first emitted token's share is p's."""
    p, q = np.array([0.5, 0.3, 0.15, 0.05]), np.array([0.1, 0.2, 0.3, 0.4])
    n, share = 200, np.zeros(4)
    for d in range(4):
        for u in (np.arange(n) + 0.5) / n:
            for w in (np.arange(20) + 0.5) / 20:
                r = speculative.verify(np.log(p)[None].repeat(2, 0), [0, d], [0, 2], [w, u], 2, np.log(q)[None].repeat(2, 0))
                share[r["token"][0, 0]] += q[d] / n / 20
    assert np.abs(share - p).max() <= 1 / n + 1 / 20 * 0.5               # a grid's resolution in either uniform


# --------------------------------------------------------------- eviction
def _evict(kw):
    b = _b()
    return _with(b.mtp_evict_args(_cache(), 10 * 2 * 4 * 16 * 64 * 2, 2, 3, 5, 40, 8, 50, 256, 512, 1024, 2048, 80, 768, 4096,
                                  1 << 20), kw)


@pytest.mark.parametrize("kw", [{"cache.pool": 0}, {"cache.head_dim": 96}, {"cache.dtype": 2}, dict(layer_stride=163832),
                                dict(layer_stride=163840 - 16), dict(n_layers=0), dict(n_layers=4097), dict(n_rows=-1),
                                dict(n_rows=4097), dict(max_pages=0), dict(max_pages=65537), dict(budget=-1, recent=-1),
                                dict(recent=-1), dict(recent=41), dict(budget=51), dict(limit=39), dict(ld=79),
                                dict(n_layers=4096, n_rows=4096), dict(table=0), dict(table=258), dict(kv_len=0),
                                dict(weights=0), dict(weights=1026), dict(out_weights=0), dict(out_len=0), dict(workspace=0),
                                dict(workspace=4096 + 128)])
def test_evict_refuses(kw):
    _refused(_b().mtp_pages_evict, _evict(kw))


def test_evict_workspace():
    b = _b()
    need = b.mtp_pages_evict_workspace_size(_evict({}))
    assert 0 < need <= 1 << 20
    _refused(b.mtp_pages_evict, _evict(dict(workspace_bytes=need - 1)), b.MTP_ENOMEM)
    with pytest.raises(b.MTPError):
        b.mtp_pages_evict_workspace_size(_evict(dict(limit=1)))
    b.mtp_pages_evict(_evict(dict(n_rows=0, table=0)), 0)
    _refused(b.mtp_pages_evict, None)


def test_oracle_eviction_of_a_hand_example():
    # 20 tokens, 6 kept, the last 2 of them recent: of the older 18 the weights 9, 8, 7, 6 at 17, 2, 9, 0
    w = np.zeros((1, 1, 1, 32), np.float32)
    w[0, 0, 0, [17, 2, 9, 0]] = 9, 8, 7, 6
    pool = np.zeros((1, 3, 2, 1, 16 * 64), np.float32)
    table = np.array([[2, 0]])
    for j in range(20):
        page = table[0, j // 16]
        pool[0, page, 0, 0].reshape(16, 64)[j % 16] = j
        pool[0, page, 1, 0].reshape(64, 16)[:, j % 16] = 100 + j
    out = np.zeros_like(w)
    n = speculative.evict(pool, True, w, table, [20], 6, 2, 6, out)
    assert n.tolist() == [6]
    want = [0, 9, 2, 17, 18, 19]                          # 0 and 2 stay; 9 and 17 fill 1 and 3; then the recent ones
    assert pool[0, 2, 0, 0].reshape(16, 64)[:6, 0].tolist() == want
    assert pool[0, 2, 1, 0].reshape(64, 16)[5, :6].tolist() == [100 + j for j in want]
    assert out[0, 0, 0, :6].tolist() == [6, 7, 8, 9, 0, 0]
    # equal weights: the first; a row within its limit stays
    out = np.zeros_like(w)
    before = pool.copy()
    assert speculative.evict(pool, True, np.ones_like(w), table, [6], 4, 1, 6, out).tolist() == [6]
    assert np.array_equal(pool, before) and out[0, 0, 0, :7].tolist() == [1] * 6 + [0]


# ------------------------------------------------------ attention weights
def _weigh(kw):
    b = _b()
    a = b.mtp_attention_args(_cache(), 2, 4, 6, 8, b.MTP_ATTN_CAUSAL, 0, 0, 0.125, 256, 512, 768, 1024, 2048, 512, 512, 4096,
                             1 << 30)
    return _with(b.mtp_weigh_args(a, 1280, 64), kw)


@pytest.mark.parametrize("kw", [{"attention.cache.pool": 0}, {"attention.n_rows": -1}, {"attention.n_heads": 6},
                                {"attention.mode": 2}, {"attention.window": -1}, {"attention.scale": NAN},
                                {"attention.max_pages": 0}, {"attention.q": 0}, {"attention.out": 2056}, {"attention.table": 0},
                                {"attention.q_stride": 504}, {"attention.workspace": 0}, {"attention.workspace": 4096 + 128},
                                dict(weights=0), dict(weights=1282), dict(ld=63)])
def test_weigh_refuses(kw):
    _refused(_b().mtp_pages_attention_weights, _weigh(kw))


def test_weigh_workspace():
    b = _b()
    need = b.mtp_pages_attention_weights_workspace_size(_weigh({}))
    assert need >= 6 * 8 * 8
    _refused(b.mtp_pages_attention_weights, _weigh({"attention.workspace_bytes": need - 1}), b.MTP_ENOMEM)
    for kw in ({"attention.n_rows": 0, "attention.table": 0}, {"attention.n_tokens": 0, "attention.q": 0}):
        assert b.mtp_pages_attention_weights_workspace_size(_weigh(kw)) == 0
        b.mtp_pages_attention_weights(_weigh(kw), 0)
    with pytest.raises(b.MTPError):
        b.mtp_pages_attention_weights_workspace_size(_weigh(dict(ld=10)))
    _refused(b.mtp_pages_attention_weights, None)


def test_oracle_weights_of_a_hand_example():
    # two keys alike: a query that sees both gives each a half, one that sees the first gives it 1
    pool = np.zeros((1, 2, 1, 16 * 64))
    w = np.full((1, 1, 16), 5.0)
    speculative.attention_weights(pool, False, np.array([[0]]), [0, 2], [3], np.ones((2, 1, 64)), w)
    assert np.allclose(w[0, 0, :3], [5 + 1 / 2 + 1 / 3, 1 / 2 + 1 / 3, 1 / 3]) and (w[0, 0, 3:] == 5).all()
    w = np.full((1, 1, 16), 5.0)
    speculative.attention_weights(pool, False, np.array([[0]]), [0, 2], [3], np.ones((2, 1, 64)), w, causal=False)
    assert np.allclose(w[0, 0, :3], 5 + 2 / 3)


STRUCTS = ["mtp_rotary", "mtp_rotate_args", "mtp_write_rotated_args", "mtp_verify_args", "mtp_evict_args", "mtp_weigh_args"]


def test_struct_layout_matches_the_header(tmp_path):
    """The ctypes structs' sizes and field offsets against the C compiler's."""
    import ctypes
    import os
    import shutil
    import subprocess
    b = _b()
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = []
    for n in STRUCTS:
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for f in getattr(b, n)._fields_]
    src = tmp_path / "layout.cpp"
    src.write_text(f'#include "{root}/include/mtp.h"\n#include <stddef.h>\n#include <stdio.h>\nint main() {{ {" ".join(lines)} }}\n')
    subprocess.run(["g++", str(src), "-o", str(tmp_path / "layout")], check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.splitlines())
    for n in STRUCTS:
        s = getattr(b, n)
        assert int(got[n]) == ctypes.sizeof(s)
        for f in s._fields_:
            assert int(got[f"{n}.{f[0]}"]) == getattr(s, f[0]).offset, (n, f[0])


def test_the_documented_bound_of_rotary_angles():
    """The reduced angle's rounding to float32 (steps of 2^-24 from 1/2 on) reaches 2^-25 and no more; float64 loses three
    roundings of 2^-53 of the turns and the constant's."""
    import os
    rng = np.random.default_rng(1)
    pos, f = rng.integers(0, 1 << 31, 1 << 20).astype(np.float64), 10000.0 ** -rng.random(1 << 20)
    t = pos * (f * 0.15915494309189533577)
    t -= np.rint(t)
    y = (4.0 * t - np.rint(4.0 * t)) * 1.57079632679489661923
    worst = np.abs(y.astype(np.float32).astype(np.float64) - y).max()
    assert np.abs(y).max() <= math.pi / 4 and 2.0 ** -26 < worst <= 2.0 ** -25
    header = open(os.path.join(os.path.dirname(__file__), "..", "include", "mtp.h")).read()
    assert "within 2^-50 of themselves and 2^-25" in header


def test_weights_workspace_follows_the_table():
    """As documented: room for the scores of every place of the table up to 256 MB, whatever the hint of the rows' length."""
    b = _b()

    def size(pages, max_kv, tokens=32):
        a = b.mtp_attention_args(b.mtp_cache(4096, b.MTP_DTYPE_BF16, 10, 8, 128), 32, pages, tokens, 32, b.MTP_ATTN_CAUSAL, 0, max_kv,
                                 0.1, 256, 256, 256, 256, 256, 4096, 4096, None, 0)
        return b.mtp_pages_attention_weights_workspace_size(b.mtp_weigh_args(a, 256, 16 * pages))

    scores = lambda pages, tokens=32: tokens * 32 * 16 * pages * 4
    for max_kv in (0, 2000):
        assert scores(125) < size(125, max_kv) and scores(1024) < size(1024, max_kv) < 2 * scores(1024)
        assert scores(4096) == 1 << 28 and size(4096, max_kv) > 1 << 28
        assert size(4097, max_kv) < 1 << 26 and size(8192, max_kv, 128) < 1 << 28
