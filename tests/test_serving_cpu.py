"""Paged serving without a GPU: the library's refusals (every one before any
launch), the argument structs' layout, and pins of the oracle's page plans."""
import ctypes
import math

import numpy as np
import pytest

from oracle import paging

INF, NAN = float("inf"), float("nan")


def _cache(**kw):
    from paper_2410_13839_amd import binding as b
    c = b.mtp_cache(4096, b.MTP_DTYPE_BF16, 10, 4, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHE = [dict(pool=0), dict(pool=4104), dict(dtype=2), dict(dtype=-1), dict(num_pages=0), dict(num_pages=1 << 27),
             dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=32), dict(head_dim=96)]


def _plan(**kw):
    from paper_2410_13839_amd import binding as b
    a = b.mtp_plan_args(2, 50000, 64, 8, None, 256, 512, 768, 1024, 2048, 2304, 2560, 2816, 3136, 3328, 4096, 1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _attention(cache=None, **kw):
    from paper_2410_13839_amd import binding as b
    a = b.mtp_attention_args(cache or _cache(), 2, 4, 6, 8, b.MTP_ATTN_CAUSAL, 0, 0, 0.125, 256, 512, 768, 1024, 2048,
                             512, 512, 4096, 1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _beam(**kw):
    from paper_2410_13839_amd import binding as b
    a = b.mtp_beam_args(2, 4, 40000, 39999, 0, 0.0, 256, 40000, 512, 768, 1024, 1280, 1536, 1792, 2048, 2304, 4096, 1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _refused(call, args, code=None):
    from paper_2410_13839_amd import binding as b
    with pytest.raises(b.MTPError) as e:
        call(args, 0)
    assert e.value.code == (b.MTP_EINVAL if code is None else code)


@pytest.mark.parametrize("kw", [dict(n_rows=-1), dict(n_rows=4097), dict(max_pages=0), dict(max_pages=65537),
                                dict(n_rows=4096, max_pages=32768), dict(num_pages=0), dict(num_pages=1 << 27),
                                dict(max_tokens=-1), dict(len=0), dict(add=0),
                                dict(table_in=0), dict(table=0), dict(row_start=0), dict(kv_len=0), dict(slots=0),
                                dict(positions=0), dict(copies=0), dict(status=0), dict(workspace=0),
                                dict(workspace=4096 + 128), dict(len=258), dict(parent=254), dict(parent=256, table=768)])
def test_plan_refuses(kw):
    from paper_2410_13839_amd import binding as b
    _refused(b.mtp_pages_plan, _plan(**kw))


def test_plan_workspace():
    from paper_2410_13839_amd import binding as b
    need = b.mtp_pages_plan_workspace_size(_plan())
    assert 0 < need <= 4096
    _refused(b.mtp_pages_plan, _plan(workspace_bytes=need - 1), b.MTP_ENOMEM)
    assert b.mtp_pages_plan_workspace_size(_plan(num_pages=1 << 20)) >= 1 << 17
    with pytest.raises(b.MTPError):
        b.mtp_pages_plan_workspace_size(_plan(num_pages=0))
    b.mtp_pages_plan(_plan(n_rows=0, len=0), 0)          # nothing to do, nothing launched


@pytest.mark.parametrize("kw", [dict(n_tokens=-1), dict(slots=0), dict(slots=258), dict(k=0), dict(k=520), dict(v=0),
                                dict(k_stride=255), dict(v_stride=248), dict(k_stride=260)])
def test_write_refuses(kw):
    from paper_2410_13839_amd import binding as b
    a = b.mtp_write_args(_cache(), 5, 256, 512, 1024, 256, 256)
    for k, v in kw.items():
        setattr(a, k, v)
    _refused(b.mtp_pages_write, a)


@pytest.mark.parametrize("kw", BAD_CACHE)
def test_bad_caches_are_refused(kw):
    from paper_2410_13839_amd import binding as b
    _refused(b.mtp_pages_write, b.mtp_write_args(_cache(**kw), 5, 256, 512, 1024, 1 << 20, 1 << 20))
    _refused(b.mtp_pages_attention, _attention(_cache(**kw)))


def test_write_and_copy_of_nothing():
    from paper_2410_13839_amd import binding as b
    b.mtp_pages_write(b.mtp_write_args(_cache(), 0, 0, 0, 0, 0, 0), 0)
    b.mtp_pages_copy(b.mtp_copy_args(4096, 4096, 40960, 2, 10, 0, 0), 0)
    b.mtp_pages_attention(_attention(n_tokens=0, q=0), 0)
    b.mtp_pages_attention(_attention(n_rows=0, table=0), 0)
    b.mtp_beam_select(_beam(n_requests=0, logits=0), 0)


@pytest.mark.parametrize("kw", [dict(pool=0), dict(pool=4104), dict(page_bytes=0), dict(page_bytes=4104),
                                dict(page_bytes=1 << 31), dict(layer_stride=40952), dict(layer_stride=36864),
                                dict(n_layers=-1), dict(n_layers=4097), dict(num_pages=0), dict(n_copies=-1),
                                dict(n_copies=4097), dict(copies=0), dict(copies=258)])
def test_copy_refuses(kw):
    from paper_2410_13839_amd import binding as b
    a = b.mtp_copy_args(4096, 4096, 40960, 2, 10, 3, 256)
    for k, v in kw.items():
        setattr(a, k, v)
    _refused(b.mtp_pages_copy, a)


@pytest.mark.parametrize("kw", [dict(n_rows=-1), dict(n_rows=4097), dict(max_pages=0), dict(max_pages=65537),
                                dict(n_tokens=-1), dict(n_tokens=1 << 24), dict(n_heads=0), dict(n_heads=6),
                                dict(n_heads=1028), dict(n_heads=1024, n_tokens=1 << 22, q_stride=1 << 16, out_stride=1 << 16), dict(mode=2), dict(mode=-1), dict(window=-1), dict(mode=1, window=5),
                                dict(max_kv=-1), dict(scale=INF), dict(scale=NAN), dict(table=0), dict(table=258),
                                dict(row_start=0), dict(kv_len=0), dict(q=0), dict(q=1032), dict(out=0), dict(out=2056),
                                dict(q_stride=504), dict(q_stride=516), dict(out_stride=511)])
def test_attention_refuses(kw):
    from paper_2410_13839_amd import binding as b
    _refused(b.mtp_pages_attention, _attention(**kw))


def test_attention_workspace():
    from paper_2410_13839_amd import binding as b
    # few rows over a long cache: the keys are split, which needs a workspace
    a = _attention(max_pages=4096)
    need = b.mtp_pages_attention_workspace_size(a)
    if need:
        a.workspace_bytes = need - 1
        _refused(b.mtp_pages_attention, a, b.MTP_ENOMEM)
        a.workspace_bytes, a.workspace = need, 4096 + 128
        _refused(b.mtp_pages_attention, a)
        a.workspace = 0
        _refused(b.mtp_pages_attention, a)
    with pytest.raises(b.MTPError):
        b.mtp_pages_attention_workspace_size(_attention(n_heads=6))


@pytest.mark.parametrize("kw", [dict(beams=0), dict(beams=33), dict(n_requests=-1), dict(n_requests=20000), dict(vocab=0),
                                dict(vocab=1 << 24), dict(eos_id=-1), dict(eos_id=40000), dict(alpha=-0.1), dict(alpha=32.5), dict(alpha=INF),
                                dict(alpha=NAN), dict(ld=39999), dict(logits=0), dict(logits=258), dict(score=0),
                                dict(len=0), dict(done=0), dict(out_score=0), dict(out_len=0), dict(out_done=0),
                                dict(out_parent=0), dict(out_token=0), dict(workspace=0), dict(workspace=4097)])
def test_beam_select_refuses(kw):
    from paper_2410_13839_amd import binding as b
    _refused(b.mtp_beam_select, _beam(**kw))


def test_beam_workspace():
    from paper_2410_13839_amd import binding as b
    need = b.mtp_beam_select_workspace_size(_beam())
    _refused(b.mtp_beam_select, _beam(workspace_bytes=need - 1), b.MTP_ENOMEM)


def test_tensors_of_the_wrong_kind_are_refused():
    torch = pytest.importorskip("torch")
    from paper_2410_13839_amd import serving
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):                       # not on a GPU
        serving.plan_pages(i, i, torch.zeros((2, 4), dtype=torch.int32), 8, 4)
    with pytest.raises(ValueError):
        serving.attend_pages(torch.zeros(4, 2, 1, 1024), i, i, i, torch.zeros(2, 1, 64))
    with pytest.raises(ValueError):
        serving._cache(torch.zeros(4, 2, 1, 1000))
    with pytest.raises(ValueError):
        serving._cache(torch.zeros(4, 2, 1, 1024, dtype=torch.float16))


# -------------------------------------------------------- the oracle's own pins
def test_oracle_plan_of_a_hand_example():
    # 2 rows: 17 cached tokens in pages 5, 2 and 3 tokens in page 0; one and 14 new ones
    table = np.array([[5, 2, -1], [0, -1, -1]], np.int32)
    r = paging.plan([17, 3], [1, 14], table, 8, 16)
    assert r["table"].tolist() == [[5, 2, -1], [0, 1, -1]]
    assert r["slots"].tolist() == [2 * 16 + 1] + [3 + i for i in range(13)] + [16] + [-1]
    assert r["positions"].tolist() == [17] + list(range(3, 17)) + [-1]
    assert r["row_start"].tolist() == [0, 1, 15] and r["kv_len"].tolist() == [18, 17]
    # both rows continue row 0: its full page is shared, row 1 gets a copy of its last one, page 0 is free again
    r = paging.plan([17, 3], [1, 1], table, 8, 2, parent=[0, 0])
    assert r["table"].tolist() == [[5, 2, -1], [5, 0, -1]]
    assert r["copies"].tolist() == [[-1, -1], [2, 0]] and r["slots"].tolist() == [33, 1]
    # a pool without room
    r = paging.plan([16, 16], [1, 17], np.array([[0, -1, -1], [1, -1, -1]]), 3, 18)
    assert r["table"].tolist() == [[0, 2, -1], [1, -1, -1]] and r["status"].tolist() == [2, 0, 0, 0]
    assert r["slots"].tolist() == [32] + [-1] * 17


def test_oracle_plan_pages_are_private():
    rng = np.random.default_rng(3)
    n, m, pages = 12, 9, 200
    table = np.full((n, m), -1, np.int32)
    length = np.zeros(n, np.int64)
    for step in range(40):
        add = rng.integers(0, 3, n)
        parent = rng.integers(0, n, n) if step % 3 == 2 else np.arange(n)
        if (length[parent] + add).max() > PAGE_LIMIT(m):
            break
        r = paging.plan(length, add, table, pages, 64, parent=parent)
        assert r["status"].tolist()[:3] == [0, 0, 0]
        table, length = r["table"], r["kv_len"].astype(np.int64)
        s = r["slots"][r["slots"] >= 0]
        assert len(set(s.tolist())) == len(s) == int(add.sum())
        for c in range(n):
            if length[c] % 16:                            # nobody else holds its last page
                last = table[c, length[c] // 16]
                assert (table == last).sum() == 1


def PAGE_LIMIT(m):
    return 16 * m


def test_oracle_beams_of_a_hand_example():
    lg = np.log(np.array([[[0.5, 0.25, 0.25], [0.1, 0.6, 0.3]]], np.float32))
    s, n, d, p, t = paging.beams(lg, np.array([[0.0, -0.1]]), np.array([[3, 3]]), np.array([[0, 0]]), 2)
    assert t.tolist() == [[1, 0]] and p.tolist() == [[1, 0]]
    assert np.allclose(s, [[math.log(0.6) - 0.1, math.log(0.5)]], atol=1e-6)
    # a finished beam keeps its score; a masked end takes no probability
    s, n, d, p, t = paging.beams(lg, np.array([[0.0, -0.1]]), np.array([[3, 3]]), np.array([[0, 1]]), 2, eos_min=4)
    assert t.tolist() == [[2, 0]] and d.tolist() == [[1, 0]] and n.tolist() == [[3, 4]]
    assert np.allclose(s, [[-0.1, math.log(0.5 / 0.75)]], atol=1e-6)


def test_struct_layout_matches_the_header(tmp_path):
    """The ctypes structs' sizes and field offsets against the C compiler's."""
    import os
    import shutil
    import subprocess
    from paper_2410_13839_amd import binding as b
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["mtp_cache", "mtp_plan_args", "mtp_write_args", "mtp_copy_args", "mtp_attention_args", "mtp_beam_args"]
    lines = []
    for n in names:
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for f in getattr(b, n)._fields_]
    src = tmp_path / "layout.cpp"
    src.write_text(f'#include "{root}/include/mtp.h"\n#include <stddef.h>\n#include <stdio.h>\nint main() {{ {" ".join(lines)} }}\n')
    subprocess.run(["g++", str(src), "-o", str(tmp_path / "layout")], check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.splitlines())
    for n in names:
        s = getattr(b, n)
        assert int(got[n]) == ctypes.sizeof(s)
        for f in s._fields_:
            assert int(got[f"{n}.{f[0]}"]) == getattr(s, f[0]).offset, (n, f[0])


def test_beam_advance_refuses_without_a_step():
    from paper_2410_13839_amd import binding as b
    from paper_2410_13839_amd.workloads import WORKLOADS
    wl = WORKLOADS["valle_k4"]
    cfg = b.make_config(wl.model, 4, wl.max_prompt, wl.max_new, wl.eos_min)
    ctx = b.mtp_create(cfg, b.mtp_buffers(256, 512, 1024, 2048), 0)
    try:
        with pytest.raises(b.MTPError) as e:
            b.mtp_beam_advance(ctx, 4, 4)
        assert e.value.code == b.MTP_ESTATE
    finally:
        b.mtp_destroy(ctx)
    assert b.mtp_query_sizes(cfg).workspace_bytes > 4 * wl.max_new * 4 * 2


def test_calls_of_more_threads_than_a_launch_holds_are_refused():
    from paper_2410_13839_amd import binding as b
    wide = dict(n_kv_heads=1024, dtype=b.MTP_DTYPE_F32)
    a = _attention(_cache(**wide), n_heads=1024, n_tokens=1 << 18, q_stride=1 << 16, out_stride=1 << 16)
    _refused(b.mtp_pages_attention, a)                   # 2^24 tiles of 16 rows
    with pytest.raises(b.MTPError):
        b.mtp_pages_attention_workspace_size(a)
    _refused(b.mtp_pages_write, b.mtp_write_args(_cache(**wide), 48 << 14, 256, 512, 1024, 1 << 16, 1 << 16))


def test_a_pool_that_needs_a_gradient_is_refused():
    torch = pytest.importorskip("torch")
    from paper_2410_13839_amd import serving
    pool = torch.zeros(4, 2, 1, 1024, requires_grad=True)
    with pytest.raises(ValueError):
        serving._cache(pool)
    with torch.no_grad():
        assert serving._cache(pool).num_pages == 4


@pytest.mark.parametrize("n_rows,n_tokens", [(0, 0), (1, 0), (2, 0), (0, 1), (0, 40)])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("dtype", [0, 1])
def test_attention_of_nothing_needs_nothing(n_rows, n_tokens, head_dim, dtype):
    from paper_2410_13839_amd import binding as b
    a = _attention(_cache(dtype=dtype, head_dim=head_dim), n_rows=n_rows, n_tokens=n_tokens, max_pages=4096)
    assert b.mtp_pages_attention_workspace_size(a) == 0
    a.workspace = a.workspace_bytes = 0
    b.mtp_pages_attention(a, 0)


@pytest.mark.parametrize("shape", [(4, 2, 1, 1024), (3, 4, 2, 1, 1024)])
def test_copies_in_pools_of_the_wrong_kind_are_refused(shape):
    torch = pytest.importorskip("torch")
    from paper_2410_13839_amd import serving
    copies = torch.full((1, 2), -1, dtype=torch.int32)
    with pytest.raises(ValueError, match="backward"):
        serving.copy_pages(torch.zeros(shape, requires_grad=True), copies)
    for dtype in (torch.float16, torch.float64, torch.int32, torch.uint8):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            serving.copy_pages(torch.zeros(shape, dtype=dtype), copies)
    for t in (torch.zeros(shape), torch.zeros(shape, dtype=torch.bfloat16)):
        with pytest.raises(ValueError, match="on a GPU"):     # (the kind is right)
            serving.copy_pages(t, copies)
    with torch.no_grad(), pytest.raises(ValueError, match="on a GPU"):
        serving.copy_pages(torch.zeros(shape, requires_grad=True), copies)


def test_tensors_with_a_tangent_are_refused():
    torch = pytest.importorskip("torch")
    from paper_2410_13839_amd import serving
    import torch.autograd.forward_ad as fwd
    pool, q, copies = torch.zeros(4, 2, 1, 1024), torch.zeros(3, 1, 64), torch.full((1, 2), -1, dtype=torch.int32)
    calls = {"pool": lambda t: serving._cache(t), "q": lambda t: serving._rows(t, "q", pool, 64),
             "pools": lambda t: serving.copy_pages(t, copies)}
    with fwd.dual_level():
        for name, t in (("pool", pool), ("q", q), ("pools", pool)):
            dual = fwd.make_dual(t, torch.ones_like(t))
            with pytest.raises(ValueError, match=f"{name}: .* forward-mode"):
                calls[name](dual)
            with torch.no_grad(), pytest.raises(ValueError, match="forward-mode"):   # (no_grad does not stop tangents)
                calls[name](dual)
        assert serving._cache(pool).num_pages == 4 and serving._rows(q, "q", pool, 64) == 64
        assert serving._cache(fwd.unpack_dual(fwd.make_dual(pool, pool)).primal).num_pages == 4

    def f(t):
        serving._rows(t, "q", pool, 64)
        return t
    with pytest.raises(ValueError, match="forward-mode"):
        torch.func.jvp(f, (q,), (q,))


def test_calls_inside_a_trace_are_refused():
    torch = pytest.importorskip("torch")
    from paper_2410_13839_amd import serving
    pool, i = torch.zeros(4, 2, 1, 1024), torch.zeros((1, 2), dtype=torch.int32)
    k, f = torch.zeros(2, 1, 64), torch.zeros(1, 2)
    calls = (lambda x: serving.plan_pages(i[0, :1], i[0, :1], i, 8, 4), lambda x: serving.write_pages(pool, i[0], k, k),
             lambda x: serving.copy_pages(pool, i), lambda x: serving.attend_pages(pool, i, i[0], i[0, :1], k),
             lambda x: serving.select_beams(torch.zeros(1, 2, 5), f, i, i, 4))
    for call in calls:
        with pytest.raises(ValueError, match="traced"):
            torch.jit.trace(lambda x: (call(x), x)[1], (f,))
        with pytest.raises(ValueError, match="on a GPU"):
            call(f)


def test_oracle_beams_that_rounding_makes_equal():
    """1e30 swallows the log probabilities: a beam's own by logit then token, the earlier beam first."""
    lg = np.array([[[0.0, 2.0, 1.0, 2.0, -INF], [5.0, 4.0, 3.0, 2.0, 1.0], [0.0, 0.0, 9.0, 0.0, 0.0]]], np.float32)
    for score, parent, token in (([-1e30, -1e30, -1e30], [0, 0, 0], [1, 3, 2]), ([-2e30, -1e30, -INF], [1, 1, 1], [0, 1, 2]),
                                 ([-INF, -INF, -1e30], [2, 2, 2], [2, 0, 1]), ([-INF, NAN, INF], [0, 0, 0], [0, 1, 2])):
        out = paging.beams(lg, np.array([score], np.float32), np.ones((1, 3)), np.zeros((1, 3)), 4)
        assert out[3].tolist() == [parent] and out[4].tolist() == [token]
