"""The dense gated delta rule against its definition in 64 bits, token by token,
and its gradients against the derivative of that definition.

Tolerance.  All products are fp32 (bf16 inputs enter exactly) and sums have at
most 256 + 64 + 64 terms: a token's row is off by at most 384 roundings of
2^-24 of the sum of its terms' magnitudes, 2.3e-5 in the worst case, and by the
root of that many, 1.2e-6, where roundings fall either way.  Errors carried in
the state shrink with it (alpha <= 1, beta |k|^2 <= 1).  1e-5 of the largest value
lies between; a wrong term or a part rounded to 16 bits (2^-9) fails it."""
import pytest
import torch

from paper_2607_07386_amd import sdm
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

TOL = 1e-5


def inputs(B, Hk, H, T, dk, dv, bf16=False, seed=0, start=True, long_memory=False):
    g = torch.Generator(device=DEV).manual_seed(seed + 131 * T + dk)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    dt = torch.bfloat16 if bf16 else torch.float32
    unit = lambda x: (x / x.norm(dim=-1, keepdim=True)).to(dt)
    a = dict(q=unit(n(B, Hk, T, dk)), k=unit(n(B, Hk, T, dk)), v=n(B, H, T, dv).to(dt),
             alpha=torch.exp(-torch.rand((B, H, T), generator=g, device=DEV) * (0.01 if long_memory else 1.5)),
             beta=torch.sigmoid(n(B, H, T)))
    return a, n(B, H, dk, dv) if start else None, n(B, H, T, dv), n(B, H, dk, dv)


def definition(a, state0, lens=None):
    """y and the last state, differentiable, in 64 bits (masked tokens change nothing)."""
    q, k, v, al, be = (a[x].double() for x in ("q", "k", "v", "alpha", "beta"))
    G = v.shape[1] // q.shape[1]
    q, k = q.repeat_interleave(G, 1), k.repeat_interleave(G, 1)
    T = v.shape[2]
    S = state0.double() if state0 is not None else v.new_zeros((*v.shape[:2], q.shape[3], v.shape[3]))
    ys = []
    for t in range(T):
        kt = k[:, :, t, :, None]
        D = al[:, :, t, None, None] * S
        new = D + kt * (be[:, :, t, None] * (v[:, :, t] - (kt * D).sum(-2)))[:, :, None]
        y = (q[:, :, t, :, None] * new).sum(-2)
        if lens is not None:
            on = (t < lens)[:, None, None]
            new, y = torch.where(on[..., None], new, S), torch.where(on, y, 0.0)
        S = new
        ys.append(y)
    return (torch.stack(ys, 2) if T else v), S


def close(got, ref, what, tol=TOL):
    ref = ref.detach()
    assert got.shape == ref.shape, what
    if ref.numel():
        e = ((got.double() - ref).abs().max() / ref.abs().max().clamp_min(1e-30)).item()
        assert e <= tol, f"{what}: {e:.2e}"


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Hk,H,T,dk,dv", [
    (1, 1, 1, 1, 4, 4), (3, 2, 4, 1, 128, 128), (2, 1, 3, 2, 36, 100), (1, 2, 2, 16, 256, 64), (2, 2, 2, 17, 128, 128), (2, 1, 2, 14, 64, 36), (2, 1, 2, 15, 64, 36),
    (1, 1, 2, 20, 256, 36), (1, 1, 2, 21, 256, 36),
    (1, 1, 2, 63, 32, 32), (1, 2, 2, 64, 64, 20), (2, 1, 1, 65, 68, 132), (1, 1, 1, 129, 4, 4), (1, 1, 2, 200, 132, 64),
    (1, 1, 1, 150, 256, 260), (2, 2, 6, 333, 96, 48),
])
def test_forward(B, Hk, H, T, dk, dv, bf16):
    a, s0, _, _ = inputs(B, Hk, H, T, dk, dv, bf16)
    for start in (None, s0):
        y, S = sdm.gdn_fwd(**a, state0=start)
        ry, rS = definition(a, start)
        close(y, ry, "y")
        close(S, rS, "state")


def test_long_memory_many_chunks():
    a, s0, _, _ = inputs(1, 1, 2, 1500, 64, 32, long_memory=True)
    y, S = sdm.gdn_fwd(**a, state0=s0)
    ry, rS = definition(a, s0)
    close(y, ry, "y")
    close(S, rS, "state")


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("dk,dv", [(16, 20), (128, 48), (132, 20), (256, 36)])
def test_few_streams_in_segments(dk, dv, bf16):
    """Long sequences of few streams run segments side by side: a full one, one that ends inside a segment,
    one that ends inside the first, one empty; with the states for a backward too."""
    T = 5 * 16 * 64 + 700
    a, s0, _, _ = inputs(4, 1, 1, T, dk, dv, bf16, long_memory=True)
    lens = torch.tensor([T, 3333, 50, 0], dtype=torch.int32, device=DEV)
    on = (torch.arange(T, device=DEV)[None] < lens[:, None])[:, None, :, None]
    ry, rS = definition(a, s0, lens)
    y, S = sdm.gdn_fwd(**a, state0=s0, lens=lens)
    close(torch.where(on, y, 0.0), ry, "y")
    close(S, rS, "state")
    saved = sdm.gdn_saved_buffer(4, 1, T, dk, dv, torch.device(DEV))
    y2, S2 = sdm.gdn_fwd(**a, state0=s0, lens=lens, saved=saved)
    assert torch.equal(y, y2) and torch.equal(S, S2)
    mine = s0.clone()
    sdm.gdn_fwd(**a, state0=mine, state_out=mine, lens=lens)
    assert torch.equal(S, mine)


def test_state_in_place_with_segments_that_some_sequences_do_not_reach():
    """More workgroups than the device holds at once, many with nothing to do but store the last state
    before the first segment's have begun: in place as into another buffer."""
    a, s0, _, _ = inputs(24, 1, 1, 5120, 128, 128, True, seed=9)
    lens = torch.tensor([5120, 100, 0, 1500] * 6, dtype=torch.int32, device=DEV)
    y, S = sdm.gdn_fwd(**a, state0=s0, lens=lens)
    for _ in range(3):
        mine = s0.clone()
        y2, S2 = sdm.gdn_fwd(**a, state0=mine, state_out=mine, lens=lens)
        assert S2 is mine and torch.equal(y, y2) and torch.equal(S, mine)
    assert torch.equal(S[2], s0[2])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,H,dk,dv", [(16, 32, 32, 32), (16, 16, 64, 32), (32, 16, 100, 32), (16, 16, 128, 36),
                                       (16, 16, 256, 32)])
def test_many_streams(B, H, dk, dv, bf16):
    """Enough column tiles for several to a workgroup, forward and backward."""
    T = 70
    a, s0, dy, dS = inputs(B, H // 2, H, T, dk, dv, bf16)
    saved = sdm.gdn_saved_buffer(B, H, T, dk, dv, torch.device(DEV))
    y, S = sdm.gdn_fwd(**a, state0=s0, saved=saved)
    y2, S2 = sdm.gdn_fwd(**a, state0=s0)
    assert torch.equal(y, y2) and torch.equal(S, S2)
    leaves = {x: t.double().requires_grad_() for x, t in a.items()}
    ls0 = s0.double().requires_grad_()
    ry, rS = definition(leaves, ls0)
    ref = torch.autograd.grad((ry, rS), [*leaves.values(), ls0], (dy.double(), dS.double()))
    close(y, ry, "y")
    close(S, rS, "state")
    g = sdm.gdn_bwd(**a, saved=saved, dy=dy, dstate_T=dS)
    for name, r in zip(("dq", "dk", "dv", "dalpha", "dbeta", "dstate0"), ref):
        close(g[name], r, name)


def test_empty_and_in_place():
    a, s0, _, _ = inputs(2, 1, 2, 0, 8, 12)
    y, S = sdm.gdn_fwd(**a, state0=s0)
    assert y.shape == (2, 2, 0, 12) and torch.equal(S, s0)
    y, S = sdm.gdn_fwd(**a)
    assert not S.any()
    for T in (1, 100):
        a, s0, _, _ = inputs(2, 1, 2, T, 24, 36)
        y, S = sdm.gdn_fwd(**a, state0=s0)
        mine = s0.clone()
        y2, S2 = sdm.gdn_fwd(**a, state0=mine, state_out=mine)
        assert S2 is mine and torch.equal(S, mine) and torch.equal(y, y2)


@pytest.mark.parametrize("T", [7, 200])
def test_padded_batch_leaves_rows_past_the_end(T):
    B, H = 5, 2
    a, s0, _, _ = inputs(B, 1, H, T, 40, 36)
    lens = torch.tensor([T, 0, 1, T // 2, T + 9], dtype=torch.int32, device=DEV)
    for b in range(B):     # what stands past a sequence's end is never read
        n = min(int(lens[b]), T)
        for x in a.values():
            x[b, :, n:] = float("nan")
    clean = {x: torch.nan_to_num(t) for x, t in a.items()}
    y0 = torch.full((B, H, T, 36), 7.5, device=DEV)
    y, S = sdm.gdn_fwd(**a, state0=s0, lens=lens, y=y0)
    ry, rS = definition(clean, s0, lens)
    on = (torch.arange(T, device=DEV)[None] < lens[:, None])[:, None, :, None]
    close(torch.where(on, y, 0.0), ry, "y")
    close(S, rS, "state")
    assert torch.all(torch.where(on, 7.5, y) == 7.5)
    assert torch.equal(S[1], s0[1])
    y, _ = sdm.gdn_fwd(**a, state0=s0, lens=lens)
    assert not torch.where(on, 0.0, y).any()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Hk,H,T,dk,dv,start", [
    (1, 1, 1, 1, 4, 4, True), (1, 1, 2, 5, 32, 32, False), (2, 1, 3, 64, 36, 100, True), (1, 2, 2, 65, 128, 128, True),
    (1, 1, 1, 130, 64, 20, False), (1, 1, 2, 90, 256, 68, True), (2, 2, 6, 193, 72, 48, True),
    (2, 2, 6, 260, 200, 48, True),
])
def test_gradients(B, Hk, H, T, dk, dv, start, bf16):
    a, s0, dy, dS = inputs(B, Hk, H, T, dk, dv, bf16, start=start)
    leaves = {x: t.double().requires_grad_() for x, t in a.items()}
    ls0 = s0.double().requires_grad_() if start else torch.zeros((B, H, dk, dv), dtype=torch.float64, device=DEV,
                                                                 requires_grad=True)
    ry, rS = definition(leaves, ls0)
    ref = torch.autograd.grad((ry, rS), [*leaves.values(), ls0], (dy.double(), dS.double()))
    saved = sdm.gdn_saved_buffer(B, H, T, dk, dv, torch.device(DEV))
    y, S = sdm.gdn_fwd(**a, state0=s0, saved=saved)
    close(y, ry, "y")
    close(S, rS, "state")
    g = sdm.gdn_bwd(**a, saved=saved, dy=dy, dstate_T=dS)
    for name, r in zip(("dq", "dk", "dv", "dalpha", "dbeta", "dstate0"), ref):
        close(g[name], r, name)


def test_gradients_against_differences():
    a, s0, dy, dS = inputs(1, 1, 2, 70, 8, 8, seed=3)
    saved = sdm.gdn_saved_buffer(1, 2, 70, 8, 8, torch.device(DEV))
    sdm.gdn_fwd(**a, state0=s0, saved=saved)
    g = sdm.gdn_bwd(**a, saved=saved, dy=dy, dstate_T=dS)

    def loss(b):
        y, S = definition(b, s0)
        return (y * dy).sum() + (S * dS).sum()

    wide = {x: t.double() for x, t in a.items()}
    for x in ("q", "k", "v", "alpha", "beta"):
        way = torch.randn(wide[x].shape, dtype=torch.float64, device=DEV)
        h = 1e-5   # central difference: off by h^2 of a third derivative, far below TOL
        d = (loss({**wide, x: wide[x] + h * way}) - loss({**wide, x: wide[x] - h * way})) / (2 * h)
        got = (g["d" + x].double() * way).sum()
        size = (g["d" + x].double() * way).abs().sum()
        assert abs(got - d) <= TOL * size, x


def test_gates_that_close():
    """alpha 0 (the memory is dropped) and tiny ones, beta 0 and 1: values and gradients."""
    a, s0, dy, dS = inputs(1, 1, 2, 140, 16, 16, seed=5)
    a["alpha"][0, 0, 10::31] = 0.0
    a["alpha"][0, 0, 30:34] = 1e-6
    a["alpha"][0, 1, 64] = 0.0
    a["beta"][0, :, 5::7] = 0.0
    a["beta"][0, 1, 6::7] = 1.0
    leaves = {x: t.double().requires_grad_() for x, t in a.items()}
    ls0 = s0.double().requires_grad_()
    ry, rS = definition(leaves, ls0)
    ref = torch.autograd.grad((ry, rS), [*leaves.values(), ls0], (dy.double(), dS.double()))
    saved = sdm.gdn_saved_buffer(1, 2, 140, 16, 16, torch.device(DEV))
    y, S = sdm.gdn_fwd(**a, state0=s0, saved=saved)
    close(y, ry, "y")
    close(S, rS, "state")
    g = sdm.gdn_bwd(**a, saved=saved, dy=dy, dstate_T=dS)
    for name, r in zip(("dq", "dk", "dv", "dalpha", "dbeta", "dstate0"), ref):
        close(g[name], r, name)


def test_gradients_of_a_padded_batch():
    B, Hk, H, T, dk, dv = 4, 1, 2, 130, 20, 24
    a, s0, dy, dS = inputs(B, Hk, H, T, dk, dv)
    lens = torch.tensor([T, 0, 64, 77], dtype=torch.int32, device=DEV)
    clean = {x: t.clone() for x, t in a.items()}
    clean_dy = dy.clone()
    for b in range(B):
        for x in (*a.values(), dy):
            x[b, :, int(lens[b]):] = float("inf")
        for x in (*clean.values(), clean_dy):
            x[b, :, int(lens[b]):] = 0.0
    leaves = {x: t.double().requires_grad_() for x, t in clean.items()}
    ls0 = s0.double().requires_grad_()
    ry, rS = definition(leaves, ls0, lens)
    ref = torch.autograd.grad((ry, rS), [*leaves.values(), ls0], (clean_dy.double(), dS.double()))
    saved = sdm.gdn_saved_buffer(B, H, T, dk, dv, torch.device(DEV))
    sdm.gdn_fwd(**a, state0=s0, lens=lens, saved=saved)
    g = sdm.gdn_bwd(**a, saved=saved, dy=dy, dstate_T=dS, lens=lens)
    for name, r in zip(("dq", "dk", "dv", "dalpha", "dbeta", "dstate0"), ref):
        close(g[name], r, name)


def test_a_sequence_in_parts_and_token_by_token():
    """The state carries: 150 tokens at once, in two calls, and one by one."""
    a, s0, _, _ = inputs(2, 1, 2, 150, 128, 128)
    y, S = sdm.gdn_fwd(**a, state0=s0)
    cut = lambda lo, hi: {x: t[:, :, lo:hi].contiguous() for x, t in a.items()}
    y1, S1 = sdm.gdn_fwd(**cut(0, 90), state0=s0)
    y2, S2 = sdm.gdn_fwd(**cut(90, 150), state0=S1)
    close(torch.cat([y1, y2], 2), y.double(), "y")
    close(S2, S.double(), "state")
    St, ys = s0.clone(), []
    for t in range(150):
        ys.append(sdm.gdn_fwd(**cut(t, t + 1), state0=St, state_out=St)[0])
    close(torch.cat(ys, 2), y.double(), "y")
    close(St, S.double(), "state")


@pytest.mark.parametrize("what", ["v", "k", "alpha"])
def test_nan_stays_in_its_heads_and_chunk_on(what):
    a, s0, _, _ = inputs(1, 2, 4, 200, 64, 32, True)
    y0, S0 = sdm.gdn_fwd(**a, state0=s0)
    a[what][0, 1, 100] = float("nan")      # v, alpha: head 1; k: the key head of heads 2 and 3
    y, S = sdm.gdn_fwd(**a, state0=s0)
    hit = [2, 3] if what == "k" else [1]
    for h in range(4):
        if h in hit:
            assert torch.equal(y[0, h, :64], y0[0, h, :64]) and torch.isnan(y[0, h, 101:]).any()
        else:
            assert torch.equal(y[0, h], y0[0, h]) and torch.equal(S[0, h], S0[0, h])


def test_same_from_run_to_run_and_on_another_stream():
    a, s0, dy, _ = inputs(2, 2, 4, 300, 128, 64, True)
    saved = sdm.gdn_saved_buffer(2, 4, 300, 128, 64, torch.device(DEV))
    y, S = sdm.gdn_fwd(**a, state0=s0, saved=saved)
    g = sdm.gdn_bwd(**a, saved=saved, dy=dy)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        saved2 = sdm.gdn_saved_buffer(2, 4, 300, 128, 64, torch.device(DEV))
        y2, S2 = sdm.gdn_fwd(**a, state0=s0, saved=saved2)
        g2 = sdm.gdn_bwd(**a, saved=saved2, dy=dy)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(S, S2)
    for x in g:
        assert torch.equal(g[x], g2[x]), x


@pytest.mark.parametrize("T", [1, 100])
def test_captured_and_replayed(T):
    a, s0, dy, _ = inputs(2, 1, 2, T, 64, 64, True)
    b, _, _, _ = inputs(2, 1, 2, T, 64, 64, True, seed=9)
    state, y = s0.clone(), torch.empty((2, 2, T, 64), device=DEV)
    saved = sdm.gdn_saved_buffer(2, 2, T, 64, 64, torch.device(DEV)) if T > 1 else None

    def step():
        sdm.gdn_fwd(**a, state0=state, state_out=state, y=y, saved=saved)
        return sdm.gdn_bwd(**a, saved=saved, dy=dy) if T > 1 else {}

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = step()
    for turn in range(3):
        for x in a:
            a[x].copy_(b[x] if turn % 2 else a[x].clone())
        state.copy_(s0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, state, *g.values())]
        state.copy_(s0)
        g2 = step()
        for x, r in zip(got, (y, state, *g2.values())):
            assert torch.equal(x, r)


def test_with_the_gates_and_the_epilogue():
    """As a layer runs it: gates from pre-activations, the rule, the gated norm, and all of it backwards."""
    B, H, T, d = 2, 3, 150, 32
    a, s0, _, _ = inputs(B, H, H, T, d, d, True)
    g = torch.Generator(device=DEV).manual_seed(1)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    a_pre, b_pre, gate, dout = n(B, H, T), n(B, H, T), n(B, H, T, d), n(B, H, T, d)
    A, b_dt, gamma = n(H).abs(), n(H), n(d)
    al, be = sdm.gates(a_pre, b_pre, A, b_dt)
    saved = sdm.gdn_saved_buffer(B, H, T, d, d, torch.device(DEV))
    y, S = sdm.gdn_fwd(a["q"], a["k"], a["v"], al, be, state0=s0, saved=saved)
    o = sdm.norm_gate(y, gate, gamma, 1e-5, 1)
    dy, dg, dgamma = sdm.norm_gate_bwd(y, gate, gamma, 1e-5, 1, dout)
    gr = sdm.gdn_bwd(a["q"], a["k"], a["v"], al, be, saved, dy)
    da, db, dA, dbd = sdm.gates_bwd(a_pre, b_pre, A, b_dt, gr["dalpha"], gr["dbeta"])
    w = [t.double().requires_grad_() for t in (a["q"], a["k"], a["v"], a_pre, b_pre, A, b_dt, gate, gamma)]
    F = torch.nn.functional
    wal = torch.exp(-w[5][:, None] * F.softplus(w[3] + w[6][:, None]))
    ry, rS = definition(dict(q=w[0], k=w[1], v=w[2], alpha=wal, beta=w[4].sigmoid()), s0)
    ro = ry * torch.rsqrt(ry.square().mean(-1, keepdim=True) + 1e-5) * w[8] * F.silu(w[7])
    ref = torch.autograd.grad(ro, w, dout.double())
    close(o, ro, "o", 2 * TOL)       # the rule's rows, then the norm's own roundings
    for name, x, r in zip(("dq", "dk", "dv", "da", "db", "dA", "db_dt", "dg", "dgamma"),
                          (gr["dq"], gr["dk"], gr["dv"], da, db, dA, dbd, dg, dgamma), ref):
        close(x, r, name, 2 * TOL)
