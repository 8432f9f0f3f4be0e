"""Packed layers on the GPU: packing, the product, its gradients and expert layers against plain 64-bit statements of their formulas.

Tolerances per element.  An output type costs half a step, eps / 2 of the value.  fp32 sums: the tensor core truncates, at most 2^-23 of the sum of the
magnitudes per instruction of 16 inputs and term, so a sum of K products is off by at most (K / 16 terms + what is added behind it) 2^-23 of
sum |x| |w|, in which a weight counts |a| |q - z| + |b + z a| because scales meet the sums afterwards.  Activations have slopes of at most 1.13 and cost
2^-20 of the value (ex2, rcp).  dX of bf16 rounds both operands: up to 2^-8 each of sum |dZ| |W|, of which the test allows 2^-8 in all."""
import pytest
import torch
import torch.nn.functional as F

from paper_2406_17542_b200 import binding as B
from paper_2406_17542_b200 import inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACTS = {"none": lambda z: z, "relu": F.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda z: F.gelu(z, approximate="tanh")}


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def make(d_in, d_out, bits, group, seed=0, lead=()):
    g = gen(seed)
    ng = d_in // (group or d_in)
    Q = torch.randint(0, 2 ** bits, (*lead, d_in, d_out), generator=g, device=DEV, dtype=torch.int64).to(torch.uint8)
    scale = 0.02 + 0.02 * torch.rand((*lead, ng, d_out), generator=g, device=DEV)
    zero = -scale * (2 ** bits - 1) / 2 * (1 + 0.1 * torch.randn((*lead, ng, d_out), generator=g, device=DEV))
    return Q, scale, zero


def weights64(Q, scale, zero):
    per = Q.shape[-2] // scale.shape[-2]
    return Q.double() * scale.double().repeat_interleave(per, -2) + zero.double().repeat_interleave(per, -2)


def magnitudes64(Q, scale, zero, bits):
    per, z = Q.shape[-2] // scale.shape[-2], 2.0 ** (bits - 1)
    s, b = scale.double().repeat_interleave(per, -2), zero.double().repeat_interleave(per, -2)
    return s.abs() * (Q.double() - z).abs() + (b + z * s).abs()


def rows(n, d, dtype, seed, pad=0):
    x = torch.randn((n, d + pad), generator=gen(seed), device=DEV).to(dtype)
    return x[:, :d]


def check(got, want, tol, what=""):
    torch.cuda.synchronize()
    assert B.load().cdq_last_device_status() == 0
    over = (got.double() - want).abs() - tol
    assert torch.isfinite(got).all() and float(over.max()) <= 0, f"{what}: {float(over.max())} over, worst at {int(over.argmax())}"


def sum_steps(K, dtype):
    return (K / 16 + 1) * (1 if dtype == torch.bfloat16 else 3) + 64


@pytest.mark.parametrize("bits", range(1, 9))
def test_packing_and_back(bits):
    for a, b in [(1, 1), (128, 16), (130, 33), (1350, 677), (127, 129), (256, 160)]:
        Q = torch.randint(0, 2 ** bits, (3, a, b), device=DEV, dtype=torch.int64).to(torch.uint8)
        one = torch.ones(3, 1, b, device=DEV)
        assert torch.equal(B.cdq_unpack(B.cdq_pack(Q, B.Grid(bits), one, one)), Q)


def product_case(n, d_in, d_out, bits, group, dtype, act, pad=0, seed=1):
    Q, scale, zero = make(d_in, d_out, bits, group, seed)
    layer = B.cdq_pack(Q, B.Grid(bits, group), scale, zero)
    X, R = rows(n, d_in, dtype, seed + 1, pad), rows(n, d_out, dtype, seed + 2, pad)
    bias = torch.randn(d_out, generator=gen(seed + 3), device=DEV)
    Y, Z = B.cdq_linear(X, layer, bias=bias, act=act, residual=R, want_z=True)
    z = X.double() @ weights64(Q, scale, zero) + bias.double()
    eps = torch.finfo(dtype).eps / 2
    err = sum_steps(d_in, dtype) * 2.0 ** -23 * (X.double().abs() @ magnitudes64(Q, scale, zero, bits) + bias.double().abs())
    check(Z, z, 1.01 * eps * z.abs() + err, "Z")
    y = ACTS[act](z)
    check(Y, y + R.double(), 1.01 * eps * (y + R.double()).abs() + 1.13 * err + 2.0 ** -20 * y.abs() + 2.0 ** -23 * R.double().abs(), "Y")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 16, 17, 33, 65, 129, 257])
@pytest.mark.parametrize("d_in,d_out,bits,group", [(256, 256, 4, 0), (1350, 677, 3, 0), (384, 100, 2, 128), (192, 130, 8, 96), (96, 40, 5, 32), (120, 50, 4, 24),
                                                   (1, 1, 1, 0), (33, 17, 3, 0), (4096, 96, 2, 256)])
def test_products(n, d_in, d_out, bits, group, dtype):
    acts = list(ACTS)
    product_case(n, d_in, d_out, bits, group, dtype, acts[(n + d_in) % len(acts)])


@pytest.mark.parametrize("n", [3, 40, 300])
def test_products_of_strided_rows(n):
    """Leading dimensions that bulk copies cannot take, and that they can."""
    for pad in (1, 8, 24):
        product_case(n, 512, 136, 4, 128, torch.bfloat16, "silu", pad)
        product_case(n, 512, 136, 4, 0, torch.float32, "gelu", pad)


@pytest.mark.parametrize("n", [4, 100])
def test_results_stay_within_their_rows_and_may_lie_on_the_residual(n):
    Q, scale, zero = make(256, 72, 3, 0)
    layer = B.cdq_pack(Q, B.Grid(3), scale, zero)
    X = rows(n, 256, torch.bfloat16, 5)
    big = torch.full((n + 2, 90), 7.0, dtype=torch.bfloat16, device=DEV)
    plain = B.cdq_linear(X, layer, residual=big[1:n + 1, 8:80])
    B.cdq_linear(X, layer, residual=big[1:n + 1, 8:80], out=big[1:n + 1, 8:80])
    assert torch.equal(big[1:n + 1, 8:80], plain)
    big[1:n + 1, 8:80] = 7.0
    assert (big == 7.0).all()


@pytest.mark.parametrize("n", [5, 60])
def test_rows_that_are_not_finite_keep_to_themselves(n):
    Q, scale, zero = make(256, 64, 4, 128)
    layer = B.cdq_pack(Q, B.Grid(4, 128), scale, zero)
    X = rows(n, 256, torch.bfloat16, 5).clone()
    good = B.cdq_linear(X, layer)
    X[1, 3], X[3, 200] = float("inf"), float("nan")
    Y = B.cdq_linear(X, layer)
    bad = torch.zeros(n, dtype=torch.bool, device=DEV)
    bad[1] = bad[3] = True
    assert torch.equal(Y[~bad], good[~bad]) and not torch.isfinite(Y[bad]).any()
    for value in (0.0, 3e38):      # all zero, and the largest magnitudes that a term can hold
        X = torch.full((n, 256), value, dtype=torch.float32, device=DEV)
        X[:, 1:] = 0
        check(B.cdq_linear(X, layer), X.double() @ weights64(Q, scale, zero), 2e38 * 2.0 ** -18)


@pytest.mark.parametrize("n", [1, 16, 100])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_graphs(n):
    Q, scale, zero = make(2048, 256, 3, 0)
    layer = B.cdq_pack(Q, B.Grid(3), scale, zero)
    X, dY = rows(n, 2048, torch.bfloat16, 5), rows(n, 256, torch.bfloat16, 6)
    both = lambda: (B.cdq_linear(X, layer, act="silu"), *B.cdq_linear_backward(dY, layer, X=X, want_bias=True).values())   # noqa: E731
    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = both()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = both()
        graphs.append((g, out))
    for g, _ in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    for other in (second, graphs[0][1], graphs[1][1]):
        assert all(torch.equal(a, b) for a, b in zip(first, other))
    X.copy_(rows(n, 2048, torch.bfloat16, 9))       # a replay reads what lies there now
    graphs[0][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(both(), graphs[0][1]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("n,d_in,d_out,bits,group", [(1, 256, 64, 4, 0), (17, 1350, 77, 3, 0), (70, 384, 200, 2, 128), (130, 192, 136, 8, 96), (300, 120, 50, 4, 24),
                                                     (257, 2048, 72, 3, 0)])
def test_gradients(n, d_in, d_out, bits, group, dtype, act):
    Q, scale, zero = make(d_in, d_out, bits, group)
    layer = B.cdq_pack(Q, B.Grid(bits, group), scale, zero)
    X, dY, Z = rows(n, d_in, dtype, 1), rows(n, d_out, dtype, 2), rows(n, d_out, dtype, 3)
    got = B.cdq_linear_backward(dY, layer, X=X, Z=Z, act=act, want_bias=True)
    dz = dY.double()
    if act != "none":
        z = Z.double().requires_grad_()
        dz, = torch.autograd.grad(ACTS[act](z), z, dz)
    W, x, ng = weights64(Q, scale, zero), X.double(), scale.shape[0]
    slope = 2.0 ** -19 * 4 if act != "none" else 0.0       # of act'(Z): four products of values good to 2^-21, magnitudes up to 4
    bdz = dz.abs() + slope * dY.double().abs()
    ddz = slope * dY.double().abs()
    eps = torch.finfo(dtype).eps / 2
    mag = bdz @ W.abs().t()
    lost = (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20) + (6 if dtype == torch.float32 else 1) * (d_out / 16 + 64) * 2.0 ** -23
    dx = dz @ W.t()
    check(got["dX"], dx, 1.01 * eps * dx.abs() + lost * mag + ddz @ W.abs().t(), "dX")
    xg, qg, zmid = x.view(n, ng, -1), Q.double().view(ng, -1, d_out), 2.0 ** (bits - 1)
    dscale = torch.einsum("nj,ngi,gij->gj", dz, xg, qg)
    dzero = torch.einsum("nj,ngi->gj", dz, xg)
    big = torch.einsum("nj,ngi,gij->gj", bdz, xg.abs(), (qg - zmid).abs() + zmid)
    per = (sum_steps(d_in // ng, dtype) + n + 64) * 2.0 ** -23
    check(got["dscale"], dscale, per * big + torch.einsum("nj,ngi,gij->gj", ddz, xg.abs(), qg), "dscale")
    check(got["dzero"], dzero, per * torch.einsum("nj,ngi->gj", bdz, xg.abs()) + torch.einsum("nj,ngi->gj", ddz, xg.abs()), "dzero")
    check(got["dbias"], dz.sum(0), (n + 8) * 2.0 ** -23 * bdz.sum(0) + ddz.sum(0), "dbias")


def test_gradients_against_differences():
    """In fp32, through the product itself: L = sum(dY * act(X W_hat + bias)), central differences in one scale, zero, bias and input at a time."""
    n, d_in, d_out = 24, 128, 48
    Q, scale, zero = make(d_in, d_out, 4, 64)
    bias = torch.randn(d_out, generator=gen(4), device=DEV)
    X, dY = rows(n, d_in, torch.float32, 1), rows(n, d_out, torch.float32, 2)
    loss = lambda layer, X, b: float((dY.double() * B.cdq_linear(X, layer, bias=b, act="silu").double()).sum())   # noqa: E731
    layer = B.cdq_pack(Q, B.Grid(4, 64), scale, zero)
    _, Z = B.cdq_linear(X, layer, bias=bias, act="silu", want_z=True)
    got = B.cdq_linear_backward(dY, layer, X=X, Z=Z, act="silu", want_bias=True)
    h = 2.0 ** -9
    W, x, d = weights64(Q, scale, zero), X.double(), dY.double()
    xq = lambda t, j: x[:, 64 * t:64 * t + 64] @ Q[64 * t:64 * t + 64, j].double()   # noqa: E731
    # (tensor, gradient, place, what the parameter is multiplied by in every z that it reaches, dY there)
    cases = [(scale, got["dscale"], (t, j), xq(t, j), d[:, j]) for t, j in [(0, 3), (1, 40)]]
    cases += [(zero, got["dzero"], (t, j), x[:, 64 * t:64 * t + 64].sum(1), d[:, j]) for t, j in [(0, 3), (1, 40)]]
    cases += [(bias, got["dbias"], (7,), torch.ones(n, dtype=torch.float64, device=DEV), d[:, 7])]
    cases += [(X, got["dX"], (r, i), W[i], d[r]) for r, i in [(0, 3), (20, 100)]]
    y = torch.nn.functional.silu(Z.double())
    for t, g, at, c, dy in cases:
        old = float(t[at])
        ends = []
        for s in (h, -h):
            t[at] = old + s
            ends.append((float(t[at]), loss(layer, X, bias)))
        t[at] = old
        slope = (ends[0][1] - ends[1][1]) / (ends[0][0] - ends[1][0])
        # a central difference is off by h^2 / 6 of the third derivative: that of silu is below 1/2, and the chain rule cubes what the parameter is
        # multiplied by.  The values are good to 2^-18 of sum |dY| (|y| + 1) at most (sums of 128 products in fp32), over 2 h
        tol = h * h / 6 * 0.5 * float((dy.abs() * c.abs() ** 3).sum()) + 2.0 ** -18 * float((d.abs() * (y.abs() + 1)).sum()) / (2 * h)
        assert abs(slope - float(g[at])) <= tol, (slope, float(g[at]), tol)


def moe64(X, router, stacks, k, act, bits):
    x = X.double()
    logits = x @ router.double()
    best, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    ids, w = ids[:, :k], torch.softmax(best[:, :k], 1)
    Y, tol = torch.zeros_like(x), torch.zeros_like(x)
    K, ff = x.shape[1], stacks[0][0].shape[-1]
    dl = (K + 64) * 2.0 ** -24 * float((x.abs() @ router.double().abs()).max())   # error of a logit
    half = 2.0 ** -16 if X.dtype == torch.bfloat16 else 2.0 ** -23
    for t in range(x.shape[0]):
        for s in range(k):
            e, xt = int(ids[t, s]), x[t]
            W = [weights64(*(v[e] for v in st)) for st in stacks]
            M = [magnitudes64(*(v[e] for v in st), bits) for st in stacks]
            g, u = xt @ W[0], xt @ W[1]
            sg = sum_steps(K, X.dtype) * 2.0 ** -23
            dg, du = sg * (xt.abs() @ M[0]), sg * (xt.abs() @ M[1])
            h = ACTS[act](g) * u
            dh = 1.13 * dg * u.abs() + (ACTS[act](g).abs() + 1.13 * dg) * du + (half + 2.0 ** -20) * h.abs()
            y = h @ W[2]
            dy = dh @ W[2].abs() + sum_steps(ff, torch.float32) * 2.0 ** -23 * (h.abs() @ M[2])
            Y[t] += w[t, s] * y
            tol[t] += w[t, s] * (dy + (2 * dl + 2.0 ** -20) * y.abs())
    return Y, tol, ids, w, dl


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d,ff,bits,group,E,k", [(1, 256, 128, 4, 0, 4, 1), (3, 130, 77, 3, 0, 5, 5), (8, 128, 384, 2, 128, 16, 2), (9, 96, 160, 8, 32, 8, 3),
                                                   (32, 256, 96, 5, 0, 2, 2), (2, 64, 64, 1, 64, 200, 16), (1, 33, 17, 4, 0, 1, 1)])
def test_expert_layers(n, d, ff, bits, group, E, k, dtype):
    stacks = [make(a, b, bits, group, 10 + i, (E,)) for i, (a, b) in enumerate([(d, ff), (d, ff), (ff, d)])]
    grid = B.Grid(bits, group)
    router = torch.randn((d, E), generator=gen(3), device=DEV).to(dtype) * (d ** -0.5)
    experts = B.PackedExperts(router, *(B.cdq_pack(Q, grid, s, z) for Q, s, z in stacks))
    X = rows(n, d, dtype, 4, 3)
    Y, ids, w = B.cdq_moe(X, experts, k, act="silu")
    want, tol, wids, ww, dl = moe64(X, router, stacks, k, "silu", bits)
    assert torch.equal(ids.long(), wids)
    check(w, ww, (2 * dl + 2.0 ** -20) * ww, "weights")
    check(Y, want, 1.01 * torch.finfo(dtype).eps / 2 * want.abs() + tol, "Y")
    again = B.cdq_moe(X, experts, k, act="silu")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured = B.cdq_moe(X, experts, k, act="silu")
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip((Y, ids, w), again, captured))


def test_equal_logits_go_to_the_lowest_experts_and_nan_to_the_last():
    d, E = 64, 40
    stacks = [make(a, b, 4, 0, i, (E,)) for i, (a, b) in enumerate([(d, 32), (d, 32), (32, d)])]
    router = torch.zeros((d, E), device=DEV)
    router[:, 5] = float("nan")
    experts = B.PackedExperts(router, *(B.cdq_pack(Q, B.Grid(4), s, z) for Q, s, z in stacks))
    _, ids, w = B.cdq_moe(rows(4, d, torch.bfloat16, 1), experts, 8)
    assert ids.tolist() == [[0, 1, 2, 3, 4, 6, 7, 8]] * 4 and torch.equal(w, torch.full_like(w, 0.125))


def test_a_quantized_layer_serves_and_is_tuned():
    """From calibration inputs to a solved layer, its packed form, its outputs, and one step on its scales that lowers the error of the outputs."""
    cfg = inputs.CONFIGS["C0"].scaled(d_in=256, d_out=96, n=512, x_dtype="bf16")
    X, W = (t.to(DEV) for t in inputs.make_layer(cfg))
    solved = B.quantize_layer(X, W, B.Grid(3, 64), passes=1, pack=True)
    layer = solved["packed"]
    assert torch.equal(B.cdq_unpack(layer), solved["Q"])
    Y = B.cdq_linear(X, layer)
    want = X.double() @ weights64(solved["Q"], solved["scale"], solved["zero"])
    mag = X.double().abs() @ magnitudes64(solved["Q"], solved["scale"], solved["zero"], 3)
    half = torch.finfo(torch.bfloat16).eps / 2      # 2^-8: eight significant bits, the last worth 2^-7, half of it lost at most
    check(Y, want, 1.01 * half * want.abs() + sum_steps(256, torch.bfloat16) * 2.0 ** -23 * mag)
    token = B.cdq_linear(X[:1], layer)
    check(token, want[:1], 1.01 * half * want[:1].abs() + sum_steps(256, torch.bfloat16) * 2.0 ** -23 * mag[:1])
    target = (X.double() @ W.double()).to(torch.bfloat16)
    grad = B.cdq_linear_backward((Y.float() - target.float()).to(torch.bfloat16), layer, X=X, want_x=False)
    e = (Y.double() - target.double())
    zslope = torch.einsum("nj,ngi->gj", e, X.double().view(512, 4, -1))
    assert float((grad["dzero"].double() * zslope).sum()) > 0
