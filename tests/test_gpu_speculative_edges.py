"""What the calls of speculative serving promise at their edges: memory that
they leave alone, and what their sums and weights mean."""
import numpy as np
import pytest

from oracle import speculative

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def serving():
    from paper_2410_13839_amd import serving as s
    return s


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a)).to(dtype).cuda()


@pytest.mark.parametrize("V,lens", [(40, [3, 1, 4]), (1025, [4]), (1025, [1]), (9000, [5, 1, 2]), (70000, [8] * 8 + [1]),
                                    (300000, [2, 3])])
def test_verify_takes_drafts_without_the_last_token_s_row(V, lens):
    """draft has a row for every token but the batch's last, whose row is not read: the drafts all pass, so that every row's
    token is drawn behind its last one."""
    from paper_2410_13839_amd import binding as b
    rng = np.random.default_rng(V)
    T, w, n = int(np.sum(lens)), max(lens), len(lens)
    logits = (rng.standard_normal((T, V)) * 2.5).astype(np.float32)
    tokens, uniforms = rng.integers(0, V, T), rng.random(T).astype(np.float32)
    start = np.concatenate([[0], np.cumsum(lens)])
    uniforms[[t for t in range(T) if t not in start]] = 0.0
    want = speculative.verify(logits, tokens, start, uniforms, w, logits)
    assert want["count"].tolist() == list(lens)
    g, u, i, rs = dev(logits, torch.float32), dev(uniforms, torch.float32), dev(tokens), dev(start)
    draft = g[:T - 1].clone()
    out = [torch.full((n, w), -7, dtype=torch.int32, device="cuda"), torch.zeros((n, w), device="cuda")] + \
        [torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(3)]
    args = b.mtp_verify_args(n, T, V, w, -1, 0, 1.0, g.data_ptr(), draft.data_ptr() if T > 1 else g.data_ptr(), V, V, i.data_ptr(),
                             rs.data_ptr(), u.data_ptr(), None, *(t.data_ptr() for t in out), None, 0)
    need = b.mtp_verify_drafts_workspace_size(args)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    if need:
        args.workspace, args.workspace_bytes = ws.data_ptr(), need
    b.mtp_verify_drafts(args, torch.cuda.current_stream().cuda_stream)
    for t, k in zip([out[0]] + out[2:], ("token", "count", "accepted", "done")):
        assert np.array_equal(t.cpu().numpy(), want[k]), k
