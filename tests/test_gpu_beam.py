"""Beam search on a context (mtp_beam_advance): the choice against the plain
selection on the GPU's own logits and scores at every step, and the logits of
the reordered rows against the float64 decoder on each row's own history, so
that states, tables and copied pages are those of the rows that are continued."""
import numpy as np
import pytest

from gpu_common import log, new_session, oracle_logits_at
from oracle import paging
from oracle.decoder import ARDecoder
from paper_2410_13839_amd.workloads import EOS_ID, VOCAB, ModelShape, Workload, make_logq, make_prompts, make_weights

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _setup(dtype, R, W, layers, d, eos_lift, phon=(2, 6), ac=(5, 30), max_new=24, eos_min=3, k_heads=2):
    shape = ModelShape(n_layers=layers, d_model=d, n_heads=d // 64, d_ff=4 * d, k_heads=k_heads, dtype=dtype, max_pos=512)
    wl = Workload("beam", shape, K=1, top_k=1, batch=R, phon_len=phon, ac_len=ac, max_new=max_new, eos_min=eos_min)
    w = make_weights(shape, seed=17)
    # an end of sequence that is likely enough to be met
    w["b_heads"] = w["b_heads"].copy()
    w["b_heads"].reshape(k_heads, VOCAB)[0, EOS_ID] += eos_lift
    pr = make_prompts(wl)
    phons = [p for p in pr.phon for _ in range(W)]
    acs = [a for a in pr.ac for _ in range(W)]
    s = new_session(wl, w, make_logq(), batch=R * W)
    s.prefill(phons, acs)
    return wl, ARDecoder(shape, w), s, phons, acs


def _search(wl, model, s, phons, acs, R, W, steps, tol, check, alpha=0.6):
    n = R * W
    hist = [[] for _ in range(n)]
    score = np.where(np.arange(n) % W == 0, 0.0, -np.inf).astype(np.float32)
    gen, done = np.zeros(n, np.int32), np.zeros(n, np.int32)
    worst = 0.0
    for i in range(steps):
        if done.all():
            break
        out = s.beam_step(W, alpha)
        lg = s.logits(1)[:, 0]
        if i in check:
            for b in range(n):
                if not done[b]:
                    ref = oracle_logits_at(model, phons[b], acs[b], hist[b], 1)[0]
                    worst = max(worst, float(np.abs(ref - lg[b]).max()))
                    assert worst <= tol, (i, b, worst)
        sc, ln, dn, par, tok = paging.beams(lg.reshape(R, W, -1), score.reshape(R, W), gen.reshape(R, W),
                                            done.reshape(R, W), EOS_ID, wl.eos_min, alpha)
        par, tok = par.reshape(-1), tok.reshape(-1)
        was = done[par] > 0
        assert np.array_equal(out["parent"], par), i
        assert np.array_equal(out["tokens"], np.where(was, -1, tok)), i
        fin = np.isfinite(sc.reshape(-1))
        assert np.abs(out["score"][fin] - sc.reshape(-1)[fin]).max() <= 2.0 ** -21 * (i + 2) + 1e-6
        hist = [list(hist[p]) + ([] if was[c] else [int(tok[c])]) for c, p in enumerate(par)]
        score, gen = out["score"], ln.reshape(-1)
        done = np.array([1 if was[c] or tok[c] == EOS_ID or len(hist[c]) >= wl.max_new else 0 for c in range(n)], np.int32)
        st = s.seq_state()
        assert np.array_equal(st["gen"], gen) and np.array_equal(st["done"], done), i
    toks = s.tokens()
    for c in range(n):
        assert toks[c][:len(hist[c])].tolist() == hist[c], c
    return hist, done, worst


@pytest.mark.parametrize("dtype,R,W,layers,d,steps,tol", [("f32", 2, 3, 2, 256, 24, 1e-4), ("f32", 1, 1, 2, 256, 6, 1e-4),
                                                          ("bf16", 2, 4, 3, 512, 40, 3e-2), ("bf16", 5, 8, 2, 512, 20, 3e-2)])
def test_beam_search_follows_the_rows_it_continues(dtype, R, W, layers, d, steps, tol):
    wl, model, s, phons, acs = _setup(dtype, R, W, layers, d, eos_lift=0.0, max_new=48)
    hist, done, worst = _search(wl, model, s, phons, acs, R, W, steps, tol, check={0, 1, 2, 7, 15, 16, 17, steps - 1})
    log(f"beam {dtype} {R} x {W}: max logit err {worst:.3g}")
    # an ordinary step of two heads after it: each row on its own history
    tok, cnt = s.step(2, 3)
    lg = s.logits(2)
    for b in range(0, R * W, max(1, R * W // 4)):
        if not done[b]:
            ref = oracle_logits_at(model, phons[b], acs[b], hist[b], 2)
            assert np.abs(ref - lg[b]).max() <= tol
    s.close()


def test_beams_end_at_eos_and_at_the_budget():
    R, W = 2, 4
    wl, model, s, phons, acs = _setup("f32", R, W, 2, 256, eos_lift=4.5, max_new=17)
    hist, done, _ = _search(wl, model, s, phons, acs, R, W, 40, 1e-4, check={1, 6, 12})
    assert done.all()
    ends = [h[-1] == EOS_ID for h in hist]
    assert any(ends), "no beam ended early"
    assert all(h[-1] == EOS_ID or len(h) == wl.max_new for h in hist)
    s.close()


def test_beam_search_is_refused_out_of_order():
    from paper_2410_13839_amd import binding as b
    wl, model, s, phons, acs = _setup("f32", 2, 2, 2, 256, 0.0)

    def refused(code, beams=2, alpha=0.0):
        with pytest.raises(b.MTPError) as e:
            b.mtp_beam_advance(s.ctx, s.B, beams, alpha)
        assert e.value.code == code

    refused(b.MTP_ESTATE)                                # no step yet
    s.step(2, 1)
    refused(b.MTP_ESTATE)                                # a step of two heads
    s.prefill(phons, acs)
    s.step(1, 1)
    for beams in (0, 3, 33, -1):
        refused(b.MTP_EINVAL, beams)
    for alpha in (-1.0, 33.0, float("nan")):
        refused(b.MTP_EINVAL, alpha=alpha)
    b.mtp_beam_advance(s.ctx, s.B, 2)
    refused(b.MTP_ESTATE)                                # twice for one step
    s.step(1, 1)
    refused(b.MTP_EINVAL, 4)                             # another number of beams
    b.mtp_beam_advance(s.ctx, s.B, 2)
    s.prefill(phons[:2] + phons[:2], [acs[0], acs[0][:-1], acs[0], acs[0]])
    s.step(1, 1)
    refused(b.MTP_EINVAL)                                # prompts of two lengths in a request
    b.mtp_beam_advance(s.ctx, s.B, 1)
    s.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_prefill_after_a_search_starts_anew(dtype):
    """The rows' shared pages, scores and states are gone: the same steps as a session that never searched, and the
    second search is the first one; two sessions' searches in turn do not meet."""
    R, W = 2, 4
    wl, model, s, phons, acs = _setup(dtype, R, W, 2, 256, 0.0)
    _, _, t, _, _ = _setup(dtype, R, W, 2, 256, 0.0)
    first = []
    for _ in range(18):
        first.append((s.beam_step(W, 0.5), s.logits(1).copy()))
    s.prefill(phons[::-1], acs[::-1])
    t.prefill(phons[::-1], acs[::-1])
    for k in (2, 1, 2, 2, 1):
        a, b = s.step(k, 2), t.step(k, 2)
        assert all(np.array_equal(x, y) for x, y in zip(a, b))
        assert np.array_equal(s.logits(k), t.logits(k))
    s.prefill(phons, acs)
    t.prefill(phons, acs)
    for out, lg in first:
        for x in (s, t):
            again = x.beam_step(W, 0.5)
            assert all(np.array_equal(again[k], out[k]) for k in out)
            assert np.array_equal(x.logits(1), lg)
    s.close()
    t.close()


def test_beam_search_after_and_between_other_calls():
    """Steps before the search, forced tokens in it, and steps of two heads behind it keep every row on its own history."""
    from paper_2410_13839_amd import binding as b
    R, W = 2, 3
    wl, model, s, phons, acs = _setup("f32", R, W, 2, 256, 0.0, max_new=40, eos_min=40)
    n = R * W
    hist = [[] for _ in range(n)]
    for _ in range(3):                                     # alike in every row of a request
        tok, cnt = s.step(2, 1)
        for c in range(n):
            hist[c] += [int(x) for x in tok[c][:cnt[c]]]
    for i in range(14):
        out = s.beam_step(W)
        hist = [list(hist[p]) + [int(out["tokens"][c])] for c, p in enumerate(out["parent"])]
        if i in (4, 9):                                    # other tokens than the chosen ones
            forced = np.array([[(7 * i + 3 * c) % 50] for c in range(n)], np.int32)
            b.mtp_force_tokens(s.ctx, forced, np.ones(n, np.int32))
            for c in range(n):
                hist[c][-1] = int(forced[c, 0])
    tok, cnt = s.step(2, 3)
    for c in range(n):
        hist[c] += [int(x) for x in tok[c][:cnt[c]]]
    s.step(1, 1)
    lg = s.logits(1)
    for c in range(n):
        if EOS_ID not in hist[c]:
            assert np.abs(oracle_logits_at(model, phons[c], acs[c], hist[c], 1)[0] - lg[c, 0]).max() <= 1e-4, c
    s.close()


@pytest.mark.parametrize("dtype,R,W,tol", [("f32", 2, 16, 1e-4), ("f32", 2, 17, 1e-4), ("f32", 1, 32, 1e-4), ("bf16", 3, 32, 3e-2)])
def test_beam_search_of_many_beams(dtype, R, W, tol):
    """Up to the 32 beams that the call takes, where the selection needs a workspace (more than 16) and where it does not."""
    wl, model, s, phons, acs = _setup(dtype, R, W, 2, 256, eos_lift=0.0, max_new=30)
    _search(wl, model, s, phons, acs, R, W, 19, tol, check={1, 18})
    s.close()
