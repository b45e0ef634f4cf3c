"""GPU: rows and weights on the 8-bit grid and the feature transform in 8-bit integers, against their definitions in 64 bits.

Codes have to be equal: the nearest whole number is decided exactly (127 x and the quotient fit 64 bits).  Products: the int32 sums are
exact, so an output is off by its few float roundings alone (u = 2^-24 each): conversion of the sum, product of the scales and with
the sum 3 u of a half, two sums 2 u of what they add; then half a step of the output's type."""
import numpy as np
import pytest
import torch

import paper_2311_06837_amd as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # the latter with room for the upper half step of a binade
F, H16 = torch.float32, torch.bfloat16


def grid(x, axis):
    """Codes and scales (float64) by the definition."""
    x = x.astype(np.float64)
    top = np.abs(x).max(axis, keepdims=True)
    bad = ~np.isfinite(x).all(axis, keepdims=True)
    live = (top >= 2.0 ** -120) & ~bad
    with np.errstate(invalid="ignore"):
        q = np.where(live, np.rint(127 * np.where(live, x, 0) / np.where(live, top, 1)), 0)
    scale = np.where(bad, np.nan, np.where(live, top / 127, 0))
    return q.astype(np.int64), scale.squeeze(axis)


def stored(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dtype)


def features(rng, M, K):
    x = rng.standard_normal((M, K)) * np.exp(rng.uniform(-3, 3, (M, 1))) * (1 + 9 * (rng.random((1, K)) < 0.02))
    x[rng.random(M) < 0.1] = 0
    return x


def on_device(a, dtype, ld=None, shift=0):
    """[M, K] in a matrix of leading dimension ld that starts `shift` elements into its allocation; NaN everywhere else."""
    M, K = a.shape
    ld = ld or K
    buf = torch.full((M * ld + shift,), float("nan"), dtype=dtype, device="cuda")
    t = buf[shift:].view(M, ld)
    t[:, :K] = stored(a, dtype).cuda()
    return t


@pytest.mark.parametrize("dtype", [F, H16])
@pytest.mark.parametrize("K", [1, 7, 16, 31, 33, 64, 100, 127, 128, 257, 602, 1000, 1031, 1500, 2047, 3001, 4096, 4097, 9001])
def test_rows(dtype, K):
    for M, listed, ld, shift, with_values in ((37, False, None, 0, True), (130, True, (K + 15) // 16 * 16 + 16, 0, False), (9, True, K + 3, 1, True)):
        print(f"rows: M={M} K={K} {dtype} listed={listed} ld={ld} shift={shift}", flush=True)
        rng = np.random.default_rng(K)
        X = on_device(features(rng, M, K), dtype, ld, shift)
        ids = rng.permutation(M)[: M // 2 + 1].astype(np.int32) if listed else None
        rows = None if ids is None else torch.from_numpy(ids).cuda()
        ldq = (K + 15) // 16 * 16 + 16
        Q = torch.full((M, ldq), 99, dtype=torch.int8, device="cuda")
        s = torch.full((M,), -5.0, device="cuda")
        V = torch.full((M, K), 7.0, dtype=dtype, device="cuda") if with_values else None
        P.gnn_quantize_rows(rows, M if ids is None else len(ids), X, K, Q, s, values=V)
        sel = np.arange(M) if ids is None else ids
        rest = np.setdiff1d(np.arange(M), sel)
        q, scale = grid(X[:, :K].float().cpu().numpy()[sel], 1)
        assert np.array_equal(Q.cpu().numpy()[sel, :K], q)
        assert not Q[torch.from_numpy(sel).long(), K:ldq - 16].any() and (Q[:, ldq - 16:] == 99).all()
        got = s.double().cpu().numpy()
        assert (np.abs(got[sel] - scale) <= U * scale).all() and (got[rest] == -5).all() and (Q[torch.from_numpy(rest).long()] == 99).all()
        if with_values:
            v = V.double().cpu().numpy()
            assert (np.abs(v[sel] - q * scale[:, None]) <= (2 * U + HALF[dtype]) * np.abs(q * scale[:, None])).all() and (v[rest] == 7).all()


def test_rows_with_infinities_nan_tiny_and_huge_values():
    x = np.ones((8, 70), dtype=np.float32)
    x[1, 3], x[2, 69], x[3, 0] = np.inf, np.nan, -np.inf
    x[4] = 1e-38          # below 2^-120
    x[5] = 3e38
    x[6] = 2.0 ** -119
    x[7] = 0
    X = torch.from_numpy(x).cuda()
    Q, s, V = torch.zeros(8, 80, dtype=torch.int8, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(8, 70, device="cuda")
    P.gnn_quantize_rows(None, 8, X, 70, Q, s, values=V)
    q, scale = grid(x, 1)
    assert np.array_equal(Q[:, :70].cpu().numpy(), q)
    assert np.allclose(s.cpu().numpy(), scale, rtol=2 * U, atol=0, equal_nan=True)
    assert torch.isnan(V[1:4]).all() and not V[4].any() and torch.isfinite(V[5:]).all()


@pytest.mark.parametrize("dtype", [F, H16])
def test_codes_next_to_borders(dtype):
    """Values one step of their type around every border between two codes, and on the borders that the type can hold."""
    tops = np.array([1.0, 127.0, 254.0, 381.0, 3.0, 0.7, 100.0, 1.9921875, 5e-30, 2e30])
    tops = stored(tops, dtype).double().numpy()
    x = (np.arange(-127, 127) + 0.5)[None] * tops[:, None] / 127
    mid = stored(x, dtype)
    # one step of the type either way: on the bit patterns, that is one up and one down in size
    pattern = torch.int32 if dtype == F else torch.int16
    both = [mid.view(pattern).add(d).view(dtype).float().numpy() for d in (-1, 0, 1)]
    x = np.concatenate(both + [tops[:, None]], 1)
    X = stored(x, dtype).cuda()
    K = x.shape[1]
    Q, s = torch.zeros(len(tops), (K + 15) // 16 * 16, dtype=torch.int8, device="cuda"), torch.zeros(len(tops), device="cuda")
    P.gnn_quantize_rows(None, len(tops), X, K, Q, s)
    assert np.array_equal(Q[:, :K].cpu().numpy(), grid(X.float().cpu().numpy(), 1)[0])


def unpack(w):
    K64, N32 = (w.K + 63) // 64 * 64, (w.N + 31) // 32 * 32
    return w.codes.view(N32 // 32, K64 // 16, 32, 16).permute(1, 3, 0, 2).reshape(K64, N32).cpu().numpy()


@pytest.mark.parametrize("dtype", [F, H16])
@pytest.mark.parametrize("K,N", [(1, 1), (16, 31), (63, 33), (64, 32), (65, 64), (129, 100), (602, 256), (257, 1031), (1500, 7)])
def test_weight(dtype, K, N):
    print(f"weight: {K} x {N} {dtype}", flush=True)
    rng = np.random.default_rng(K + N)
    W = on_device(features(rng, N, K).T.copy(), dtype, N + 5 if K % 2 else None)[:, :N]
    V = torch.zeros(K, N, dtype=dtype, device="cuda")
    w = P.gnn_quantize_weight(W, values=V)
    q, scale = grid(W.float().cpu().numpy(), 0)
    full = unpack(w)
    assert np.array_equal(full[:K, :N], q) and not full[K:].any() and not full[:, N:].any()
    assert (np.abs(w.scale.double().cpu().numpy() - scale) <= U * scale).all()
    assert (np.abs(V.double().cpu().numpy() - q * scale) <= (2 * U + HALF[dtype]) * np.abs(q * scale)).all()
    again = P.gnn_quantize_weight(W, out=w)
    assert again is w and np.array_equal(unpack(w), full)


@pytest.mark.parametrize("dtype", [F, H16])
def test_values_in_the_place_of_the_input(dtype):
    for M, K in ((70, 602), (5, 9000)):
        X = torch.randn(M, K, device="cuda").to(dtype)
        Q, s, V = torch.zeros(M, (K + 15) // 16 * 16, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda"), torch.zeros_like(X)
        P.gnn_quantize_rows(None, M, X, K, Q, s, values=V)
        P.gnn_quantize_rows(None, M, X, K, Q, s, values=X)
        assert torch.equal(X, V)
    W, V = torch.randn(300, 70, device="cuda").to(dtype), torch.zeros(300, 70, dtype=dtype, device="cuda")
    P.gnn_quantize_weight(W, values=V)
    P.gnn_quantize_weight(W, values=W)
    assert torch.equal(W, V)


def test_weight_column_with_nan():
    W = torch.randn(100, 40, device="cuda")
    W[99, 7], W[0, 33] = float("nan"), float("inf")
    w = P.gnn_quantize_weight(W)
    bad = torch.isnan(w.scale)
    assert bad.nonzero().flatten().tolist() == [7, 33] and not unpack(w)[:, [7, 33]].any()


def product(M, K, N, src, kind, out, relu, listed, bias=True, seed=0, shift=0, ldh=None, pad=0):
    """One call, checked against the definition; kind: "i8", F or H16."""
    print(f"product: M={M} K={K} N={N} src={src} in={kind} out={out} relu={relu} listed={listed}", flush=True)
    rng = np.random.default_rng(seed + 7 * M + K + 13 * N)
    ld = (K + 15) // 16 * 16 + 16 * pad if kind == "i8" else K + pad
    total, mass = np.zeros((M, N)), np.zeros((M, N))
    args, ws = [], []
    for _ in range(src):
        if kind == "i8":
            q = rng.integers(-127, 128, (M, K))
            s = rng.random(M).astype(np.float32) * np.float32(0.02)
            q[0], q[-1] = 127, -127          # the largest sums
            t = torch.full((M, ld), 77, dtype=torch.int8, device="cuda")   # what lies beyond K must not count
            t[:, :K] = torch.from_numpy(q.astype(np.int8)).cuda()
            args += [t, torch.from_numpy(s).cuda()]
        else:
            x = on_device(features(rng, M, K), kind, ld, shift)
            q, s = grid(x[:, :K].float().cpu().numpy(), 1)
            args += [x, None]
        W = rng.standard_normal((K, N)).astype(np.float32)
        W[:, 0] = 1.0
        w = P.gnn_quantize_weight(torch.from_numpy(W).cuda())
        wq, wsc = grid(W, 0)
        ws.append(w)
        half = (q.astype(np.float64) @ wq.astype(np.float64)) * s[:, None].astype(np.float64) * wsc      # sums of whole numbers below 2^53: exact
        total += half
        mass += np.abs(half)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    if bias:
        total += b
        mass += np.abs(b)
    if relu:
        total = np.maximum(total, 0)
    if src == 1:
        args += [None, None]
    ids = rng.permutation(M)[: M // 2 + 1].astype(np.int32) if listed else None
    rows = None if ids is None else torch.from_numpy(ids).cuda()
    H = torch.full((M, ldh or N), 5.0, dtype=out, device="cuda")
    P.gnn_linear_i8_fwd(rows, M if ids is None else len(ids), args[0], args[1], args[2], args[3], K, ws[0], ws[1] if src == 2 else None,
                        torch.from_numpy(b).cuda() if bias else None, H, relu)
    sel = np.arange(M) if ids is None else ids
    got = H.double().cpu().numpy()
    # scales are floats here and exact quotients in the reference: 2 u more a half; sums of two halves and the bias 2 u
    err = 8 * U * mass[sel] + HALF[out] * np.abs(total[sel]) + 1e-300
    assert (np.abs(got[sel, :N] - total[sel]) <= err).all(), np.max(np.abs(got[sel, :N] - total[sel]) / err)
    rest = np.setdiff1d(np.arange(M), sel)
    assert (got[rest] == 5).all() and (got[:, N:] == 5).all()


@pytest.mark.parametrize("kind", ["i8", F, H16])
@pytest.mark.parametrize("src", [1, 2])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 602, 256), (3, 64, 32), (16, 65, 33), (17, 128, 41), (33, 129, 100), (127, 192, 129), (128, 256, 128),
                                   (129, 300, 47), (300, 602, 256), (257, 1031, 300), (64, 2100, 70), (1000, 16, 8), (40, 4100, 48), (70, 1000, 64), (100, 641, 300), (63, 1024, 65),
                                   (200, 577, 96), (65, 255, 257)])
def test_product(kind, src, M, K, N):
    out = F if (M + K) % 2 else H16
    product(M, K, N, src, kind, out, relu=N % 2 == 0, listed=K % 2 == 1, bias=M != 3, ldh=N + 3 if M % 2 else None, pad=M % 3, shift=1 if M == 300 else 0)


@pytest.mark.parametrize("kind", ["i8", F, H16])
@pytest.mark.parametrize("out", [F, H16])
def test_product_many_rows(kind, out):
    product(5003, 602, 256, 2, kind, out, True, True)
    product(40_001, 128, 64, 1, kind, out, False, False)


@pytest.mark.parametrize("src", [1, 2])
@pytest.mark.parametrize("M,K,N", [(33, 1100, 200), (300, 1025, 129), (2100, 1091, 2050), (6200, 1088, 2049), (40_000, 1025, 65), (6100, 641, 2050)])
def test_product_tiles_of_every_size(M, K, N, src):
    """Reductions over 1024, and codes: few tiles of 64, of 128 (256 of them and more), of 256 (192 and more, one source)."""
    product(M, K, N, src, "i8", F if K % 2 else H16, N % 2 == 0, M == 2100)
    if M < 3000:
        product(M, K, N, src, H16, H16, N % 2 == 0, M == 300)


@pytest.mark.parametrize("kind", ["i8", F, H16])
@pytest.mark.parametrize("K,N,src", [(608, 512, 2), (640, 513, 2), (600, 1000, 2), (1024, 160, 2), (1000, 96, 1), (256, 600, 1), (31, 544, 2), (640, 65, 1)])
def test_product_panels(K, N, src, kind):
    """Tiles of 32 and 64 rows, one panel and several, more tiles than compute units and fewer."""
    for M in (50, 1700, 17_000):
        if M * N < 6_000_000:
            product(M, K, N, src, kind, H16 if N % 32 == 0 else F, True, M == 1700, pad=8 if kind != "i8" and K % 8 == 0 else 0)


def test_a_rows_answer_does_not_depend_on_the_others():
    """The same bits whether a row is asked for alone, with few, with many, and whichever way its codes come."""
    X = torch.randn(17_000, 608, device="cuda").to(H16)
    X[:, 602:] = 0
    w = [P.gnn_quantize_weight(torch.randn(602, 300, device="cuda")) for _ in range(2)]
    bias = torch.randn(300, device="cuda")
    Q, s = torch.zeros(17_000, 608, dtype=torch.int8, device="cuda"), torch.zeros(17_000, device="cuda")
    P.gnn_quantize_rows(None, 17_000, X, 602, Q, s)
    outs = []
    for M in (1, 20, 40, 1000, 17_000):
        for x, sc in ((X, None), (Q, s)):
            H = torch.zeros(M, 300, device="cuda")
            P.gnn_linear_i8_fwd(None, M, x, sc, x, sc, 602, w[0], w[1], bias, H, True)
            outs.append(H)
    for H in outs:
        assert torch.equal(H, outs[-1][: H.shape[0]])


@pytest.mark.parametrize("K,N,src,sizes", [
    (1091, 300, 1, (1, 20, 40, 1000, 11_000, 25_000)),      # few rows, then tiles of 64, of 128 (256 tiles of them), of 256 (192)
    (1091, 300, 2, (1, 20, 40, 1000, 11_000)),              # two sources: tiles of 64 and 128
    (602, 50, 1, (1, 20, 40, 1000, 33_000, 50_000)),        # codes of narrow outputs take the tiles, floats the panels
    (602, 50, 2, (1, 20, 40, 1000, 33_000)),
])
@pytest.mark.parametrize("kind", [F, H16])
def test_a_rows_answer_is_the_same_in_every_kernel(kind, K, N, src, sizes):
    """Equal to the bit, from rows and from codes, with the neighbour half, the vertex's own, bias and ReLU; listed rows of the largest
    size too."""
    print(f"every kernel: K={K} N={N} src={src} {kind}", flush=True)
    M, Kq = sizes[-1], (K + 15) // 16 * 16
    X = [torch.randn(M, Kq, device="cuda").to(kind) for _ in range(src)]
    w = [P.gnn_quantize_weight(torch.randn(K, N, device="cuda")) for _ in range(src)] + [None]
    bias = torch.randn(N, device="cuda")
    Q = [torch.zeros(M, Kq, dtype=torch.int8, device="cuda") for _ in range(src)]
    s = [torch.zeros(M, device="cuda") for _ in range(src)]
    for k in range(src):
        P.gnn_quantize_rows(None, M, X[k], K, Q[k], s[k])

    def answer(rows, n, codes):
        x, sc = (Q, s) if codes else (X, [None] * src)
        H = torch.full((M, N), 7.0, device="cuda")
        P.gnn_linear_i8_fwd(rows, n, x[0], sc[0], x[1] if src == 2 else None, sc[1] if src == 2 else None, K, w[0], w[1], bias, H, True)
        return H
    want = answer(None, M, True)
    for codes in (True, False):
        for n in sizes:
            H = answer(None, n, codes)
            assert torch.equal(H[:n], want[:n]) and (H[n:] == 7).all(), (codes, n)
        n = M - M // 50      # a list that still fills the largest tiles
        ids = torch.randperm(M, device="cuda")[:n].to(torch.int32)
        H = answer(ids, n, codes)
        there = torch.zeros(M, dtype=torch.bool, device="cuda")
        there[ids.long()] = True
        assert torch.equal(H[there], want[there]) and (H[~there] == 7).all(), codes


def test_product_long_reduction():
    product(65, 65536, 40, 1, "i8", F, False, False)
    product(2, 20_000, 33, 2, H16, F, False, False)


@pytest.mark.parametrize("M", [1, 20, 200, 3000])
@pytest.mark.parametrize("kind", ["i8", F, H16])
def test_product_of_bad_rows_stays_in_them(M, kind):
    """A row with a NaN (a scale of NaN, for codes) gives a row of NaN, through the ReLU too; a row of zeros gives the bias."""
    K, N = 100, 50
    X = torch.randn(M, K, device="cuda")
    X[M // 2, 3] = float("nan")
    w = P.gnn_quantize_weight(torch.randn(K, N, device="cuda"))
    bias = torch.rand(N, device="cuda")
    if M > 2:
        X[M - 1] = 0
    args = X.to(H16) if kind == H16 else X
    scale = None
    if kind == "i8":
        args, scale = torch.zeros(M, 112, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda")
        P.gnn_quantize_rows(None, M, X, K, args, scale)
    H = torch.zeros(M, N, device="cuda")
    P.gnn_linear_i8_fwd(None, M, args, scale, None, None, K, w, None, bias, H, True)
    assert torch.isnan(H[M // 2]).all() and torch.isnan(H).sum() == N
    if M > 2:
        assert torch.equal(H[M - 1], bias)


def test_product_is_the_same_whichever_way_the_codes_come():
    for M in (5, 700):
        X = torch.randn(M, 602, device="cuda")
        w, w2 = (P.gnn_quantize_weight(torch.randn(602, 100, device="cuda")) for _ in range(2))
        Q, s = torch.zeros(M, 608, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda")
        P.gnn_quantize_rows(None, M, X, 602, Q, s)
        outs = []
        for x, sc in ((X, None), (Q, s)):
            H = torch.zeros(M, 100, device="cuda")
            P.gnn_linear_i8_fwd(None, M, x, sc, x, sc, 602, w, w2, None, H, False)
            outs.append(H)
        assert torch.equal(*outs)


def test_product_in_a_graph():
    X, w = torch.randn(500, 300, device="cuda"), P.gnn_quantize_weight(torch.randn(300, 64, device="cuda"))
    H, ws = torch.zeros(500, 64, device="cuda"), P.Workspace()
    call = lambda: P.gnn_linear_i8_fwd(None, 500, X, None, None, None, 300, w, None, None, H, True, ws=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        X.normal_()
        g.replay()
        got = H.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, H)


def test_rows_beyond_32_bits():
    """Rows whose first element lies beyond 2^31: codes from them, and products of them by every route."""
    M, K, N = 2_200_000, 1024, 40
    X = torch.zeros(M, K, dtype=H16, device="cuda")
    X[-500:] = torch.randn(500, K, device="cuda").to(H16)
    Q, s = torch.zeros(M, K, dtype=torch.int8, device="cuda"), torch.zeros(M, device="cuda")
    ids = torch.arange(M - 500, M, dtype=torch.int32, device="cuda")
    P.gnn_quantize_rows(ids, 500, X, K, Q, s)
    near, ns = torch.zeros(500, K, dtype=torch.int8, device="cuda"), torch.zeros(500, device="cuda")
    P.gnn_quantize_rows(None, 500, X[-500:], K, near, ns)
    assert torch.equal(Q[-500:], near) and torch.equal(s[-500:], ns) and not Q[:1000].any()
    w = P.gnn_quantize_weight(torch.randn(K, N, device="cuda"))
    want = torch.zeros(500, N, device="cuda")
    P.gnn_linear_i8_fwd(None, 500, near, ns, None, None, K, w, None, None, want, False)
    H = torch.zeros(M, N, device="cuda")
    for x, sc in ((X, None), (Q, s)):
        for n in (20, 500):
            H[-500:] = 0
            P.gnn_linear_i8_fwd(ids[-n:].contiguous(), n, x, sc, None, None, K, w, None, None, H, False)
            assert torch.equal(H[-n:], want[-n:]) and not H[-500:-n].any()
