"""det_verify_drafts against a plain implementation in extended precision: accepted counts and tokens have to be equal."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, step, up

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def d():
    import paper_2602_00182_amd as d
    return d


def plain(p, q, drafts, n, u):
    B, N = drafts.shape
    V = p.shape[2]
    accepted, tokens = np.zeros(B, np.int32), np.full((B, N + 1), -1, np.int32)
    for b in range(B):
        a, m = 0, min(max(int(n[b]), 0), N)
        while a < m and 0 <= drafts[b, a] < V:
            x = drafts[b, a]
            qx = np.longdouble(1) if q is None else np.longdouble(q[b, a, x])
            if not np.longdouble(u[b, a]) * qx < np.longdouble(p[b, a, x]):
                break
            tokens[b, a] = x
            a += 1
        target = p[b, a].astype(np.longdouble)
        left = target.copy()
        if a < m:
            if q is None:
                if 0 <= drafts[b, a] < V:
                    left[drafts[b, a]] = 0
            else:
                left = target - q[b, a].astype(np.longdouble)
        left = np.where(left > 0, left, 0)
        if not left.any():
            left = np.where(target > 0, target, 0)
        sums = np.cumsum(left)
        past = np.flatnonzero(sums > np.longdouble(u[b, N]) * sums[-1])
        accepted[b] = a
        tokens[b, a] = past[0] if len(past) else (np.flatnonzero(left)[-1] if left.any() else 0)
    return accepted, tokens


def softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


def check(d, p, q, drafts, n, u, name):
    B, N = drafts.shape
    accepted = torch.full((B,), 77, dtype=torch.int32, device=DEV)
    tokens = torch.full((B, N + 1), 77, dtype=torch.int32, device=DEV)
    step(name)
    d.det_verify_drafts(up(p), None if q is None else up(q), up(drafts), None if n is None else up(n), up(u), accepted, tokens)
    torch.cuda.synchronize()
    want = plain(p, q, drafts, np.full(B, N) if n is None else n, u)
    assert np.array_equal(accepted.cpu().numpy(), want[0])
    assert np.array_equal(tokens.cpu().numpy(), want[1])
    return want


@pytest.mark.parametrize("V", [1, 2, 15, 64, 1000, 1027, 4096, 32003, 128000])
@pytest.mark.parametrize("N", [1, 4, 63])
def test_random_drafts(d, V, N):
    B = 5 if V * N < 2000000 else 2
    rng = np.random.default_rng(V * 64 + N)
    logits = 3 * rng.standard_normal((B, N + 1, V))
    p, q = softmax(logits), softmax(logits[:, :N] + 0.2 * rng.standard_normal((B, N, V)))
    drafts = (logits[:, :N] + rng.gumbel(size=(B, N, V))).argmax(-1).astype(np.int32)
    n = rng.integers(0, N + 1, B).astype(np.int32)
    n[0] = N
    u = rng.random((B, N + 1), dtype=np.float32)
    check(d, p, q, drafts, n, u, f"V {V} N {N}")
    check(d, p, None, drafts, None, u, f"V {V} N {N}, certain drafts")


def test_every_draft_accepted_and_none(d):
    rng = np.random.default_rng(5)
    B, N, V = 6, 5, 3001
    p = softmax(rng.standard_normal((B, N + 1, V)))
    drafts = rng.integers(0, V, (B, N)).astype(np.int32)
    u = rng.random((B, N + 1), dtype=np.float32)
    zero, one = u.copy(), u.copy()
    zero[:, :N] = 0.0
    want = check(d, p, p[:, :N].copy(), drafts, None, zero, "all accepted")
    assert (want[0] == N).all()
    sure = np.zeros((B, N, V), np.float32)
    np.put_along_axis(sure, drafts[..., None], 1.0, 2)
    one[:, :N] = 1 - 2.0 ** -24
    want = check(d, p, sure, drafts, None, one, "none accepted")
    assert (want[0] == 0).all()
    assert (want[1] == check(d, p, None, drafts, None, one, "the same, certain drafts")[1]).all()


def test_borders(d):
    """Sums that are exact in any order: a target on a border belongs to the next token; equality does not accept."""
    V = 4099
    p = np.zeros((4, 2, V), np.float32)
    p[:, :, [3, 700, 701, 4098]] = 0.25
    q = np.zeros((4, 1, V), np.float32)
    q[:, :, 3] = 0.5
    drafts = np.full((4, 1), 3, np.int32)
    u = np.array([[0.5, 0.0], [0.5, 1 / 3], [0.5, 0.999], [0.49999997, 0.75]], np.float32)
    want = check(d, p, q, drafts, None, u, "borders")
    assert want[0].tolist() == [0, 0, 0, 1] and want[1][:, 0].tolist() == [700, 701, 4098, 3] and want[1][3, 1] == 4098


def test_rows_with_nothing_left_and_rows_that_are_no_probabilities(d):
    V, N = 515, 2
    p = np.full((7, N + 1, V), 1 / 512, np.float32)
    q = np.full((7, N, V), 1 / 256, np.float32)      # p - q is negative everywhere: the token comes from p
    drafts = np.full((7, N), 9, np.int32)
    p[1] = 0                                         # nothing anywhere: token 0
    p[2, 0, :] = np.nan
    p[2, 0, 44] = 0.5                                # NaN counts 0 and accepts nothing
    drafts[3] = [-1, 600]                            # ids that are none
    q[4, 0, 9] = np.nan
    p[5, 0] = 0
    p[5, 0, 514] = 1e-30                             # what is left lies in the last token
    q[5, 0] = 0
    q[5, 0, 9] = 1
    p[6, 0] = -p[6, 0]
    n = np.array([2, 2, 2, 2, 2, 2, -4], np.int32)
    u = np.full((7, N + 1), 0.75, np.float32)
    want = check(d, p, q, drafts, n, u, "odd rows")
    assert want[1][1, 0] == 0 and want[1][2, 0] == 44 and want[1][5, 0] == 514
    check(d, p, None, drafts, n, u, "odd rows, certain drafts")


def test_many_parts_and_few_tokens_that_count(d):
    """Rows of several hundred parts in which nearly all tokens weigh nothing: whatever the target, a token that weighs something is drawn."""
    rng = np.random.default_rng(9)
    B, V = 40, 700001
    p = np.zeros((B, 2, V), np.float32)
    for b in range(B):
        at = rng.integers(0, V, 3)
        p[b, :, at] = rng.random((3, 1), dtype=np.float32) + np.float32(1e-3)
    q = np.zeros((B, 1, V), np.float32)
    drafts = rng.integers(0, V, (B, 1)).astype(np.int32)
    u = rng.random((B, 2), dtype=np.float32)
    u[:4, 1] = [0.0, 1 - 2.0 ** -24, 0.5, 1e-30]
    want = check(d, p, q, drafts, None, u, "few tokens that count")
    assert all(p[b, 0, want[1][b, 0]] > 0 for b in range(B) if want[0][b] == 0)


def test_graph_replays(d):
    rng = np.random.default_rng(8)
    B, N, V = 3, 3, 32000
    p, q = softmax(rng.standard_normal((B, N + 1, V))), softmax(rng.standard_normal((B, N, V)))
    drafts, u = rng.integers(0, V, (B, N)).astype(np.int32), rng.random((B, N + 1), dtype=np.float32)
    want = plain(p, q, drafts, [N] * B, u)
    dev = [up(x) for x in (p, q, drafts, u)]
    accepted, tokens = torch.empty(B, dtype=torch.int32, device=DEV), torch.empty((B, N + 1), dtype=torch.int32, device=DEV)
    run = lambda: d.det_verify_drafts(dev[0], dev[1], dev[2], None, dev[3], accepted, tokens)
    run()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            run()
    for _ in range(3):
        accepted.fill_(9)
        tokens.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(accepted.cpu().numpy(), want[0]) and np.array_equal(tokens.cpu().numpy(), want[1])
