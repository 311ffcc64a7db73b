"""The projections against fp64, forward and backward, flat and head-major.

Tolerance, relative to the largest value.  fp32: a sum of n terms is off by at most
n roundings of 2^-24 of the terms' magnitudes together, whose sum is at most about
sqrt(n) times the result's largest value for terms of either sign: sqrt(n) n 2^-24 in
the worst case, n 2^-24 where roundings fall either way (4e-5 at n = 700); activations add
a few roundings.  bf16: inputs are exact, sums as before, and one rounding of the result,
2^-8 at most; gradients enter through dz rounded to bf16 as well, at most 2^-8 of each
term, so of the sum of magnitudes: 2^-8 sqrt(n) in the worst case, and 2^-8 where they
fall either way.  Twice 2^-8 covers both roundings.  An fp32 x rounded to bf16 counts
like dz."""
import pytest
import torch

from paper_2607_07386_amd import sdm
from tests.gpu_util import DEV

pytestmark = pytest.mark.gpu

F32_TOL, BF16_TOL = 4e-5, 2 * 2.0 ** -8
ACTS = [lambda z: z, torch.nn.functional.silu, torch.nn.functional.gelu]


def close(got, ref, what, tol):
    ref = ref.detach()
    assert got.shape == ref.shape, what
    if ref.numel():
        e = ((got.double() - ref).abs().max() / ref.abs().max().clamp_min(1e-30)).item()
        assert e <= tol, f"{what}: {e:.2e}"


def flat(x):
    return x.transpose(1, 2).flatten(-2) if x.dim() == 4 else x


def case(B, T, K, N, hin, hout, bf16, x_f32=False, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + B * T + K + N)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = n(B, hin, T, K // hin) if hin else n(B, T, K)
    return (x if x_f32 else x.to(dt), (n(N, K) / K ** 0.5).to(dt), n(N), n(B, T, N).to(dt),
            (n(B, hout, T, N // hout) if hout else n(B, T, N)).to(dt))


def reference(x, w, bias, act, residual, hout):
    z = flat(x) @ w.T
    z = z if bias is None else z + bias
    y = ACTS[act](z)
    y = y if residual is None else y + residual
    to = lambda a: a.unflatten(-1, (hout, -1)).transpose(1, 2) if hout else a
    return to(y), to(z)


SHAPES = [  # B, T, K, N, heads in, heads out
    (1, 1, 8, 1, 0, 0), (3, 1, 64, 7, 0, 7), (16, 1, 256, 512, 0, 4), (2, 33, 40, 130, 5, 0), (1, 129, 136, 65, 0, 5),
    (2, 257, 96, 96, 2, 3), (1, 300, 704, 260, 0, 0), (3, 50, 520, 24, 13, 12), (1, 640, 512, 512, 8, 8),
    (5, 1, 1024, 1, 0, 0), (2, 512, 256, 384, 2, 6), (1, 1, 4096, 300, 0, 0), (1, 64, 72, 40, 3, 2), (1, 65, 72, 32, 0, 4),
    (3, 50, 72, 33, 9, 0), (2, 65, 200, 64, 5, 4), (1, 33, 1000, 50, 0, 0),
]


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed", "bf16_to_f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, kind, act):
    B, T, K, N, hin, hout = shape
    bf = kind != "f32"
    x, w, bias, res, _ = case(B, T, K, N, hin, hout, bf, kind == "mixed")
    out = torch.float32 if kind == "bf16_to_f32" else None
    tol = F32_TOL if kind in ("f32", "bf16_to_f32") else BF16_TOL
    for b in (None, bias):
        for r in (None, res) if not hout else (None,):
            r = r if r is None or out is None else r.float()
            y, z = sdm.linear(x, w, b, act=act, residual=r, heads=hout, out_dtype=out, want_z=True)
            ry, rz = reference(x.double(), w.double(), None if b is None else b.double(), act,
                               None if r is None else r.double(), hout)
            assert y.dtype == (out or w.dtype)
            close(y, ry, "y", tol)
            close(z, rz, "z", tol)
    assert torch.equal(y, sdm.linear(x, w, b, act=act, residual=r, heads=hout, out_dtype=out))


@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed", "bf16_dy_f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients(shape, kind, act):
    B, T, K, N, hin, hout = shape
    bf = kind != "f32"
    x, w, bias, _, dy = case(B, T, K, N, hin, hout, bf, kind == "mixed")
    if kind == "bf16_dy_f32":
        dy = dy.float() * 1.001
    y, z = sdm.linear(x, w, bias, act=act, heads=hout, want_z=True)
    g = sdm.linear_bwd(x, w, dy, z=z if act else None, act=act, want_dbias=True)
    # the derivative at the z that was kept (its rounding is the forward's, not the gradients')
    zd = flat(z.double()).requires_grad_()
    dz, = torch.autograd.grad(ACTS[act](zd), zd, flat(dy.double()))
    dz = dz.flatten(0, 1)
    xd = flat(x.double()).flatten(0, 1)
    dx = (dz @ w.double()).view(B, T, K)
    dx = dx.unflatten(-1, (hin, -1)).transpose(1, 2) if hin else dx
    tol = BF16_TOL if bf else F32_TOL
    assert g["dx"].dtype == x.dtype and g["dw"].dtype == w.dtype
    close(g["dx"], dx, "dx", tol)
    close(g["dw"], dz.T @ xd, "dw", tol)
    close(g["dbias"], dz.sum(0), "dbias", F32_TOL)
    g2 = sdm.linear_bwd(x, w, dy, z=z, act=act, want_dx=False)
    assert g2["dx"] is None and g2["dbias"] is None and torch.equal(g2["dw"], g["dw"])
    g3 = sdm.linear_bwd(x, w, dy, z=z, act=act, want_dw=False)
    assert torch.equal(g3["dx"], g["dx"])


@pytest.mark.parametrize("shape", [(3, 40, 64, 48, 0, 0), (2, 700, 40, 33, 0, 11), (1, 5, 64, 64, 4, 8)])
def test_bias_gradient_at_the_unrounded_z(shape):
    """With what z's rounding left, the slope is the fp32 one's to 2^-17 of z (|z act''| <= 1), and dbias an fp32 sum."""
    B, T, K, N, hin, hout = shape
    x, w, bias, _, dy = case(B, T, K, N, hin, hout, True)
    for act in (1, 2):
        y, z, rest = sdm.linear(x, w, bias, act=act, heads=hout, want_z=True, want_rest=True)
        ry, rz = reference(x.double(), w.double(), bias.double(), act, None, hout)
        close(z, rz, "z", BF16_TOL)
        close(z.double() + rest.double(), rz, "z + rest", F32_TOL)
        g = sdm.linear_bwd(x, w, dy, z=z, z_rest=rest, act=act, want_dbias=True)
        zd = flat(rz).detach().requires_grad_()
        dz, = torch.autograd.grad(ACTS[act](zd), zd, flat(dy.double()))
        close(g["dbias"], dz.flatten(0, 1).sum(0), "dbias", F32_TOL)
    assert sdm.linear(x.float(), w.float(), act=1, want_z=True, want_rest=True)[2] is None


def test_gradients_against_differences():
    x, w, bias, _, dy = case(2, 20, 16, 12, 0, 3, False)
    for act in (1, 2):
        _, z = sdm.linear(x, w, bias, act=act, heads=3, want_z=True)
        g = sdm.linear_bwd(x, w, dy, z=z, act=act, want_dbias=True)
        at = dict(x=x.double(), w=w.double(), bias=bias.double())
        loss = lambda a: (reference(a["x"], a["w"], a["bias"], act, None, 3)[0] * dy).sum()
        for name in at:
            way = torch.randn_like(at[name])
            d = (loss({**at, name: at[name] + 1e-5 * way}) - loss({**at, name: at[name] - 1e-5 * way})) / 2e-5
            got = g["d" + name].double() * way
            assert abs(got.sum() - d) <= F32_TOL * got.abs().sum(), name


@pytest.mark.parametrize("heads", [0, 8])
def test_more_than_2_gib(heads):
    """1,049,000 rows of 1024 bf16 values: offsets within x, and within dy, that pass 31 bits (rows flat, heads
    head-major).  Gradients whose dy is zero but for a few rows need only those."""
    M, K, N = 1049000, 1024, 64
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randint(-8, 9, (M, K), generator=g, device=DEV, dtype=torch.int8).to(torch.bfloat16) / 8
    w = (torch.randint(-8, 9, (N, K), generator=g, device=DEV) / 64).to(torch.bfloat16)
    assert x.numel() * 2 > 2 ** 31
    at = torch.tensor([0, 1, 255, 256, M // 2, M - 300, M - 2, M - 1], device=DEV)
    rows, wd = x[at].double(), w.double()
    lay = (lambda t: t.view(1, M, heads, -1).transpose(1, 2).contiguous()) if heads else (lambda t: t[None])
    xl = lay(x)
    y = sdm.linear(xl, w, out_dtype=torch.float32)
    close(y[0, at], rows @ wd.T, "y", F32_TOL)
    dy = torch.zeros((1, M, N), dtype=torch.bfloat16, device=DEV)
    dy[0, at] = (torch.randint(-8, 9, (len(at), N), generator=g, device=DEV) / 8).to(torch.bfloat16)
    del y
    out = sdm.linear_bwd(xl, w, dy)
    close(out["dw"], dy[0, at].double().T @ rows, "dw", BF16_TOL)
    dx = out["dx"].transpose(1, 2)[0, at].flatten(1) if heads else out["dx"][0, at]
    close(dx, dy[0, at].double() @ wd, "dx", BF16_TOL)
    del out, dx
    # the other way round: the 1024 values are the outputs (wide dy)
    wt = w.T.contiguous()
    out = sdm.linear_bwd(dy, wt, xl)
    close(out["dx"][0, at], rows @ wd.T, "dx of wide outputs", BF16_TOL)
    close(out["dw"], rows.T @ dy[0, at].double(), "dw of wide outputs", BF16_TOL)


def test_bias_gradient_of_many_tokens():
    """9,000,000 tokens: more blocks of 128 rows than a grid takes in one direction.  Terms of one sign, each
    in at most 144 / 8 + 8 + 65,535 / 32 + 32 additions: off by 2106 roundings of 2^-24 of the sum at most."""
    M, N = 9000000, 8
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.ones((1, M, 8), dtype=torch.bfloat16, device=DEV)
    w = torch.eye(8, dtype=torch.bfloat16, device=DEV)
    dy = torch.rand((1, M, N), generator=g, device=DEV) + 0.5
    out = sdm.linear_bwd(x, w, dy, want_dw=False, want_dbias=True)
    close(out["dbias"], dy[0].double().sum(0), "dbias", 2106 * 2.0 ** -24)
    close(out["dx"][0, -1000:], dy[0, -1000:].double(), "dx", 2 * 2.0 ** -8)


@pytest.mark.parametrize("K,hin", [(136, 0), (68, 17), (2048, 8)])
@pytest.mark.parametrize("N", [1, 16, 17, 33, 64, 65])
@pytest.mark.parametrize("M", [127, 129, 256, 257, 5000])
def test_weights_gradient_with_few_outputs(M, N, K, hin):
    """Tokens that end inside a group of 128 and inside a part; what lies past the end of x's last row is not
    read into a sum.  5000 terms of either sign: see the module's tolerance (5000 2^-24 is 3e-4 in the worst
    case of roundings that all fall one way; they fall either way)."""
    x, w, _, _, dy = case(1, M, K, N, hin, 0, False)
    out = sdm.linear_bwd(x, w, dy, want_dx=False)
    close(out["dw"], flat(dy.double()).flatten(0, 1).T @ flat(x.double()).flatten(0, 1), "dw", F32_TOL)


def test_no_tokens():
    w, b = torch.randn(24, 16, device=DEV), torch.randn(24, device=DEV)
    x = torch.empty((2, 0, 16), device=DEV)
    assert sdm.linear(x, w, b).shape == (2, 0, 24)
    g = sdm.linear_bwd(x, w, torch.empty((2, 0, 24), device=DEV), want_dbias=True)
    assert g["dx"].shape == x.shape and not g["dw"].any() and not g["dbias"].any()


def test_infinities_stay_in_their_rows():
    """A row's infinity or NaN touches no other row (and no padding of a tile gets in)."""
    x, w, bias, _, _ = case(1, 70, 64, 40, 0, 0, True)
    y0 = sdm.linear(x, w, bias)
    x[0, 5, 3], x[0, 69, 0] = float("inf"), float("nan")
    y = sdm.linear(x, w, bias)
    keep = [i for i in range(70) if i not in (5, 69)]
    assert torch.equal(y[:, keep], y0[:, keep])
    assert not torch.isfinite(y[0, 5]).any() and torch.isnan(y[0, 69]).all()


def test_in_place_residual_stream_and_graph():
    B, T, K, N = 2, 100, 128, 96
    x, w, bias, res, dy = case(B, T, K, N, 0, 0, True)
    y = sdm.linear(x, w, bias, act=1, residual=res)
    mine = res.clone()
    sdm.linear(x, w, bias, act=1, residual=mine, y=mine)
    assert torch.equal(mine, y)
    xs = x.clone()

    def step():
        y, z = sdm.linear(xs, w, bias, act=1, residual=res, want_z=True)
        return dict(y=y, **sdm.linear_bwd(xs, w, dy, z=z, act=1, want_dbias=True))

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = step()
    for turn in range(3):
        xs.copy_(x * (turn + 1))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {a: t.clone() for a, t in g.items()}
        for a, t in step().items():
            assert torch.equal(t, got[a]), a


def test_layer_from_stream_to_stream():
    """x -> projections (head-major) -> gates -> dense rule -> gated norm -> output projection + residual,
    and back, as a layer chains them; fp32, against the derivative in 64 bits."""
    B, T, D, H, d = 2, 100, 48, 3, 16
    g = torch.Generator(device=DEV).manual_seed(0)
    n = lambda *s: torch.randn(s, generator=g, device=DEV)
    x, dout = n(B, T, D), n(B, T, D)
    wq, wk, wv, wg = (n(H * d, D) / D ** 0.5 / 2 for _ in range(4))
    wa, wb, wo = n(H, D) / D ** 0.5, n(H, D) / D ** 0.5, n(D, H * d) / (H * d) ** 0.5
    A, b_dt, gamma = n(H).abs(), n(H), n(d)
    q, k, v, gate = (sdm.linear(x, w, heads=H) for w in (wq, wk, wv, wg))
    k = k * 0.25      # so that beta |k|^2 stays small and the update contracts
    a_pre, b_pre = (sdm.linear(x, w, heads=H)[..., 0].contiguous() for w in (wa, wb))
    al, be = sdm.gates(a_pre, b_pre, A, b_dt)
    saved = sdm.gdn_saved_buffer(B, H, T, d, d, torch.device(DEV))
    y, _ = sdm.gdn_fwd(q, k, v, al, be, saved=saved)
    o = sdm.norm_gate(y, gate, gamma, 1e-5, 1)
    out = sdm.linear(o, wo, residual=x)
    go = sdm.linear_bwd(o, wo, dout)
    dy, dgate, _ = sdm.norm_gate_bwd(y, gate, gamma, 1e-5, 1, go["dx"])
    gr = sdm.gdn_bwd(q, k, v, al, be, saved, dy)
    da, db, _, _ = sdm.gates_bwd(a_pre, b_pre, A, b_dt, gr["dalpha"], gr["dbeta"])
    dx, dws = dout.clone(), {}
    for name, w, grad in (("q", wq, gr["dq"]), ("k", wk, gr["dk"] * 0.25), ("v", wv, gr["dv"]), ("g", wg, dgate),
                          ("a", wa, da[..., None].contiguous()), ("b", wb, db[..., None].contiguous())):
        s = sdm.linear_bwd(x, w, grad)
        dx += s["dx"]
        dws[name] = s["dw"]
    leaves = [t.double().requires_grad_() for t in (x, wq, wk, wv, wg, wa, wb, wo)]
    X, WQ, WK, WV, WG, WA, WB, WO = leaves
    F = torch.nn.functional
    split = lambda z: z.unflatten(-1, (H, -1)).transpose(1, 2)
    Q, K_, V, Gt = split(X @ WQ.T), split(X @ WK.T) * 0.25, split(X @ WV.T), split(X @ WG.T)
    al_ = torch.exp(-A.double()[:, None] * F.softplus((X @ WA.T).transpose(1, 2) + b_dt.double()[:, None]))
    be_ = (X @ WB.T).transpose(1, 2).sigmoid()
    S, ys = torch.zeros((B, H, d, d), dtype=torch.float64, device=DEV), []
    for t in range(T):
        kt = K_[:, :, t, :, None]
        Dm = al_[:, :, t, None, None] * S
        S = Dm + kt * (be_[:, :, t, None] * (V[:, :, t] - (kt * Dm).sum(-2)))[:, :, None]
        ys.append((Q[:, :, t, :, None] * S).sum(-2))
    Y = torch.stack(ys, 2)
    O = Y * torch.rsqrt(Y.square().mean(-1, keepdim=True) + 1e-5) * gamma.double() * F.silu(Gt)
    ref = O.transpose(1, 2).flatten(-2) @ WO.T + X
    grads = torch.autograd.grad(ref, leaves, dout.double())
    # five operators one after the other, each within F32_TOL of its own inputs
    tol = 5 * F32_TOL
    close(out, ref, "out", tol)
    close(dx, grads[0], "dx", tol)
    for name, r in zip("qkvgab", grads[1:7]):
        close(dws[name], r, "dw" + name, tol)
    close(go["dw"], grads[7], "dwo", tol)
