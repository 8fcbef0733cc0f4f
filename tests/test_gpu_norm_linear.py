"""Layer norm, 8-bit rows and the 8-bit linear layer on the GPU, through the binding, against the float64 oracle.

Tolerances.  u = 2^-24: half a step of f32.  A sum of n terms in any order is off by at most n u of the sum of magnitudes (2 n u where an adder cuts instead of
rounding, as a matrix unit may).  The 8-bit matrix unit, which products with bf16 outputs use, cuts each of eight products that it adds at a time at 2^-13 of the largest's power of
two: at most 8 * 2^-13 of the sum of magnitudes.  A value stored in bf16 by half a step, 2^-8 of it (torch.finfo(bf16).eps / 2).  Packing and restoring are exact."""
import numpy as np
import pytest
import torch

from oracle import norm_linear_oracle as orc
from paper_2603_16435_amd import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
CUT = {"f32": 0.0, "bf16": 8 * 2.0 ** -13}


def half_step(dtype, v):
    return torch.finfo(dtype).eps / 2 * np.abs(v) * (1 + 2.0 ** -7) + 1e-38


def f64(t):
    return t.double().cpu().numpy()


def rows(a, dtype, pad=0, device="cuda"):
    """a on the GPU, as columns of a buffer that is `pad` columns wider."""
    t = torch.full((a.shape[0], a.shape[1] + pad), 7.0, dtype=dtype)
    t[:, :a.shape[1]] = torch.from_numpy(a).to(dtype)
    return t.to(device)[:, :a.shape[1]]


def state(rng, R, H):
    x = rng.normal(size=(R, H)) * np.exp(rng.normal(size=(R, 1))) * (1 + 30 * (rng.random(H) < 0.02)) + 0.5 * rng.normal(size=H)
    if R > 4:
        x[3] = 0                                                     # a padding row
        x[4, : H // 2] = 0                                           # blocks of zeros
    return x


# ------------------------------------------------------------------ layer norm
NORM = [(1, 1), (3, 7), (5, 64), (2, 127), (9, 128), (6, 130), (4, 512), (37, 513), (5, 1000), (300, 768), (11, 1157), (3, 2048), (7, 2051), (6, 4096), (5, 5120),
        (3, 8192), (4, 8200), (2, 16384), (2100, 96), (2055, 1157), (2049, 2304), (2050, 4096)]


@pytest.mark.parametrize("R, H", NORM + [(1025, 1025), (1030, 1536), (1100, 1283)])
@pytest.mark.parametrize("dtype, params, kept, pad", [("bf16", "f32", None, 0), ("bf16", "bf16", "e4m3", 5), ("f32", "f32", "e5m2", 0), ("f32", "bf16", None, 3)])
def test_layer_norm(R, H, dtype, params, kept, pad):
    rng = np.random.default_rng(R * 31 + H)
    t = DT[dtype]
    x = rows(state(rng, R, H), t, pad)
    dy = rows(rng.normal(size=(R, H)) * (rng.random((R, 1)) < 0.8) * 1e-3, t, pad)
    gamma, beta = (torch.from_numpy(1 + 0.3 * rng.normal(size=H)).to(DT[params]).cuda(), torch.from_numpy(0.2 * rng.normal(size=H)).to(DT[params]).cuda())
    y, stats, ckpt = binding.rl_layer_norm_forward(x, gamma, beta, eps=1e-5, checkpoint=kept)
    xs = f64(x)
    ry, mean, rstd = orc.norm_forward(xs, f64(gamma), f64(beta), 1e-5)
    n = 100                                                          # roundings on the way of a value through a row's sum: 64 in a lane, 6 + 16 between them
    ma = np.abs(xs).mean(1, keepdims=True)
    xh = (xs - mean) * rstd
    U_xh = n * U * (3 * ma * rstd + 3 * np.abs(xh) + 3 * ma ** 2 * rstd ** 2 * n * U * np.abs(xh))          # of the mean, and of rstd
    tol = U_xh * np.abs(f64(gamma)) + 3 * U * (np.abs(ry) + np.abs(f64(beta))) + half_step(t, ry)
    assert np.all(np.abs(f64(y) - ry) <= tol), np.max(np.abs(f64(y) - ry) / tol)
    assert np.all(np.abs(f64(stats)[:, :1] - mean) <= n * U * ma + 1e-38)
    if kept:
        want, es = orc.round_rows(xs, kept)
        assert np.array_equal(f64(binding.rl_f8_unpack(ckpt, torch.float32)), want)
        assert np.array_equal(ckpt.scales[:, :es.shape[1]].cpu().numpy().astype(int) - 127, es)
        again = binding.rl_f8_pack(x, kept)
        assert torch.equal(again.codes, ckpt.codes) and torch.equal(again.scales, ckpt.scales)
        xs = want
    # backward, from the statistics that the forward pass returned
    mean, rstd = f64(stats)[:, :1], f64(stats)[:, 1:]
    d = f64(dy)
    rdx, rdg, rdb = orc.norm_backward(d, xs, mean, rstd, f64(gamma))
    dx, dg, db = binding.rl_layer_norm_backward(dy, ckpt if kept else x, stats, gamma)
    xh, g = (xs - mean) * rstd, d * f64(gamma)
    e_xh = 3 * U * (np.abs(xs) + np.abs(mean)) * rstd
    s_g, s_gx = np.abs(g).mean(1, keepdims=True), np.abs(g * xh).mean(1, keepdims=True)
    tol = rstd * (4 * U * np.abs(g) + n * U * s_g + np.abs(xh) * (n * U * s_gx + (np.abs(g) * e_xh).mean(1, keepdims=True)) + e_xh * s_gx + 4 * U * np.abs(xh) * s_gx) + half_step(t, rdx)
    assert np.all(np.abs(f64(dx) - rdx) <= tol), np.max(np.abs(f64(dx) - rdx) / tol)
    tol = (R + 3) * U * np.abs(d * xh).sum(0) + (np.abs(d) * e_xh).sum(0) + 1e-38
    assert np.all(np.abs(f64(dg) - rdg) <= tol), np.max(np.abs(f64(dg) - rdg) / tol)
    assert np.all(np.abs(f64(db) - rdb) <= R * U * np.abs(d).sum(0) + 1e-38)
    assert torch.all(dx[(dy == 0).all(1)] == 0)                      # a row without a gradient
    # the same bits again; in place; without beta's gradient
    dx2, dg2, none = binding.rl_layer_norm_backward(dy.clone() if pad == 0 else dy, ckpt if kept else x, stats, gamma, want_beta=False)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2) and none is None
    same, _, _ = binding.rl_layer_norm_backward(dy, ckpt if kept else x, stats, gamma, out=dy)
    assert torch.equal(same, dx) and same.data_ptr() == dy.data_ptr()
    y2, _, _ = binding.rl_layer_norm_forward(x, gamma, beta, eps=1e-5, out=x)
    assert torch.equal(y2, y)
    if pad:                                                          # and what lies between the rows stays
        assert torch.all(x._base[:, H:] == 7) and torch.all(dy._base[:, H:] == 7)


@pytest.mark.parametrize("R, H", [(1, 5), (200, 4096), (512, 1157), (512, 16384), (700, 1000), (1300, 1157)])
@pytest.mark.parametrize("over", ["dy", "x", "kept"])
def test_layer_norm_backward_in_place_keeps_the_sums(R, H, over):
    """dx over dy (or x): the sums over the rows are those of dy and x as they came."""
    rng = np.random.default_rng(R + H)
    x, dy = rows(rng.normal(size=(R, H)), torch.bfloat16, 0), rows(rng.normal(size=(R, H)), torch.bfloat16, 0)
    gamma = torch.from_numpy(rng.normal(size=H).astype(np.float32)).cuda()
    _, stats, kept = binding.rl_layer_norm_forward(x, gamma, checkpoint="e4m3" if over == "kept" else None)
    dx, dg, db = binding.rl_layer_norm_backward(dy, kept or x, stats, gamma)
    out = x if over == "x" else dy
    dx2, dg2, db2 = binding.rl_layer_norm_backward(dy, kept or x, stats, gamma, out=out)
    assert dx2.data_ptr() == out.data_ptr() and torch.equal(dx, dx2) and torch.equal(dg, dg2) and torch.equal(db, db2)


def test_layer_norm_without_beta_and_without_rows():
    x = torch.randn(3, 40, device="cuda")
    gamma = torch.randn(40, device="cuda")
    zero = torch.zeros(40, device="cuda")
    assert torch.equal(binding.rl_layer_norm_forward(x, gamma)[0], binding.rl_layer_norm_forward(x, gamma, zero)[0])
    e = x[:0]
    y, stats, kept = binding.rl_layer_norm_forward(e, gamma, checkpoint="e4m3")
    assert y.shape == (0, 40) and kept.codes.shape == (0, 128)
    dx, dg, db = binding.rl_layer_norm_backward(e, kept, stats, gamma)
    assert dx.shape == (0, 40) and torch.all(dg == 0) and torch.all(db == 0)


def test_layer_norm_keeps_what_is_not_finite_in_its_row():
    rng = np.random.default_rng(5)
    x = rng.normal(size=(9, 700))
    x[2, 5], x[4, 699], x[7, 0] = np.inf, np.nan, -np.inf
    t = rows(x, torch.bfloat16)
    gamma = torch.ones(700, device="cuda")
    y, stats, kept = binding.rl_layer_norm_forward(t, gamma, checkpoint="e4m3")
    bad = np.zeros(9, bool)
    bad[[2, 4, 7]] = True
    assert np.array_equal(~np.isfinite(f64(y)).all(1), bad)
    dy = rows(rng.normal(size=(9, 700)), torch.bfloat16)
    dx, _, db = binding.rl_layer_norm_backward(dy, kept, stats, gamma)
    assert np.array_equal(~np.isfinite(f64(dx)).all(1), bad) and torch.isfinite(db).all()
    # a constant row: variance zero
    c = torch.full((2, 700), 3.0, device="cuda")
    y, stats, _ = binding.rl_layer_norm_forward(c, gamma, eps=1e-5)
    assert torch.all(y.abs() <= 700 * U * 3 * 320) and torch.isfinite(stats).all()


@pytest.mark.parametrize("R, H", [(1, 3), (5, 64), (40, 1157), (700, 1000), (600, 2304), (530, 5120), (1500, 1283)])
@pytest.mark.parametrize("dtype, fmt", [("bf16", None), ("bf16", "e4m3"), ("f32", None), ("f32", "e5m2")])
def test_layer_norm_rows_without_a_gradient_contribute_nothing(R, H, dtype, fmt):
    """dy zero where x is infinite or no number: the gradients are those with such rows of x zero."""
    rng = np.random.default_rng(R + H)
    x, dy = rng.normal(size=(R, H)), rng.normal(size=(R, H))
    bad = rng.random(R) < 0.3
    bad[-1] = True
    dy[bad] = 0
    clean = x.copy()
    clean[bad] = 0
    x[bad, rng.integers(0, H, size=bad.sum())] = rng.choice([np.inf, -np.inf, np.nan], size=bad.sum())
    gamma = torch.from_numpy(rng.normal(size=H).astype(np.float32)).cuda()
    got = []
    for v in (x, clean):
        t, d = rows(v, DT[dtype]), rows(dy, DT[dtype])
        _, stats, kept = binding.rl_layer_norm_forward(t, gamma, checkpoint=fmt)
        got.append(binding.rl_layer_norm_backward(d, kept or t, stats, gamma))
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


# ------------------------------------------------------------------ 8-bit rows
@pytest.mark.parametrize("R, K", [(1, 1), (3, 127), (2, 128), (5, 129), (4, 512), (3, 513), (7, 1157), (2, 2048), (2, 2050), (6, 5120), (70, 300)])
@pytest.mark.parametrize("dtype, fmt, pad", [("bf16", "e4m3", 0), ("bf16", "e5m2", 3), ("f32", "e4m3", 1), ("f32", "e5m2", 0)])
def test_pack_is_exact(R, K, dtype, fmt, pad):
    rng = np.random.default_rng(R + K)
    x = state(rng, R, K) * 10.0 ** rng.integers(-20, 20, size=(R, 1))
    if R > 1 and K > 100:
        x[1, 3], x[1, 50], x[1, 99], x[1, 64] = np.inf, -np.inf, np.nan, -0.0
    x[0, 0] = 448.0
    t = rows(x, DT[dtype], pad)
    p = binding.rl_f8_pack(t, fmt)
    want, es = orc.round_rows(f64(t), fmt)
    got = f64(binding.rl_f8_unpack(p, torch.float32))
    assert np.array_equal(got, want, equal_nan=True), np.argwhere((got != want) & ~np.isnan(want))[:4]
    assert np.array_equal(np.signbit(got[~np.isnan(got)]), np.signbit(want[~np.isnan(want)]))
    assert np.array_equal(p.scales[:, :es.shape[1]].cpu().numpy().astype(int) - 127, es)
    assert torch.all(p.scales[:, es.shape[1]:] == 127) and torch.all(p.codes[:, K:] & 0x7f == 0)
    back = binding.rl_f8_unpack(p, DT[dtype])
    assert torch.equal(torch.nan_to_num(back.float(), nan=3.0), torch.nan_to_num(torch.from_numpy(want).float().to(DT[dtype]).float(), nan=3.0).cuda())


def test_pack_every_value_and_tie_of_the_format():
    for fmt in ("e4m3", "e5m2"):
        v = orc.values(fmt)
        a = np.concatenate([v, (v[1:] + v[:-1]) / 2, np.nextafter(((v[1:] + v[:-1]) / 2).astype(np.float32), np.float32(1e9))])
        a = np.concatenate([a, -a])
        x = np.full((len(a), 128), v[-1])                            # one value under test a block, the largest beside it: scale 1
        x[:, 7] = a
        got = f64(binding.rl_f8_unpack(binding.rl_f8_pack(rows(x, torch.float32), fmt), torch.float32))
        want, _ = orc.round_rows(x.astype(np.float32).astype(np.float64), fmt)
        assert np.array_equal(got, want)


def test_pack_at_the_ends_of_the_range():
    x = np.zeros((6, 256))
    x[0, :128], x[1, :128], x[2, :128] = 3.4e38, 1e-38, 2.0 ** -140
    x[3, 5], x[4, 5], x[5, 130] = 2.0 ** -149, 448 * 2.0 ** -127, -3.4028234663852886e38
    x[1, 3], x[2, 3] = 1e-40, 2.0 ** -149
    for fmt in ("e4m3", "e5m2"):
        t = rows(x, torch.float32)
        want, es = orc.round_rows(f64(t), fmt)
        p = binding.rl_f8_pack(t, fmt)
        assert np.array_equal(p.scales[:, :2].cpu().numpy().astype(int) - 127, es)
        assert np.array_equal(f64(binding.rl_f8_unpack(p, torch.float32)), want)


@pytest.mark.parametrize("N, K", [(1, 1), (5, 130), (128, 128), (129, 127), (200, 515), (384, 256)])
@pytest.mark.parametrize("dtype, fmt", [("f32", "e4m3"), ("bf16", "e5m2")])
def test_weight_and_its_transpose_hold_the_same_values(N, K, dtype, fmt):
    rng = np.random.default_rng(N * K)
    w = rows(rng.normal(size=(N, K)) * np.exp(2 * rng.normal(size=(N, 1))), DT[dtype], pad=1)
    p = binding.rl_f8_pack_weight(w, fmt)
    want = orc.round_weight(f64(w), fmt)
    assert np.array_equal(f64(binding.rl_f8_unpack(p.rows, torch.float32)), want)
    assert np.array_equal(f64(binding.rl_f8_unpack(p.cols, torch.float32)), want.T)
    assert torch.all(p.rows.codes[:, K:] & 0x7f == 0) and torch.all(p.cols.codes[:, N:] & 0x7f == 0)
    assert torch.equal(binding.rl_f8_pack_weight(w, fmt, transposed=False).rows.codes, p.rows.codes)


# ------------------------------------------------------------------ products
MATMUL = [(1, 1, 1), (1, 16, 128), (2, 5, 130), (16, 33, 257), (16, 100, 4500), (17, 64, 128), (17, 65, 300), (64, 64, 513), (100, 130, 1157), (129, 257, 640),
          (70, 50, 5000), (300, 200, 2300), (257, 256, 384), (513, 260, 129)]


@pytest.mark.parametrize("M, N, K", MATMUL)
@pytest.mark.parametrize("fa, fb, dtype", [("e4m3", "e4m3", "f32"), ("e5m2", "e4m3", "bf16"), ("e4m3", "e5m2", "f32"), ("e5m2", "e5m2", "bf16")])
def test_matmul(M, N, K, fa, fb, dtype):
    rng = np.random.default_rng(M + N + K)
    a = binding.rl_f8_pack(rows(state(rng, M, K) * 2.0 ** rng.integers(-9, 9, size=(M, 1)), torch.float32), fa)
    b = binding.rl_f8_pack_weight(rows(rng.normal(size=(N, K)) / K ** 0.5, torch.float32), fb).rows
    y = binding.rl_f8_matmul(a, b, DT[dtype])
    va, vb = f64(binding.rl_f8_unpack(a, torch.float32)), f64(binding.rl_f8_unpack(b, torch.float32))
    want = va @ vb.T
    tol = (2 * (K + 32) * U + CUT[dtype]) * (np.abs(va) @ np.abs(vb).T) + half_step(DT[dtype], want)
    assert np.all(np.abs(f64(y) - want) <= tol), np.max(np.abs(f64(y) - want) / tol)
    assert np.linalg.norm(f64(y) - want) <= 2.0 ** -8 * np.linalg.norm(want)
    if dtype == "f32":                                               # and no less exact than adding in f32 is: a random walk of K roundings, four times over
        walk = U * np.sqrt(K + 32) * np.sqrt((va ** 2) @ (vb ** 2).T) * 4 + U * np.abs(want)
        assert np.linalg.norm(f64(y) - want) <= 4 * np.linalg.norm(walk)
    assert torch.equal(y, binding.rl_f8_matmul(a, b, DT[dtype]))


def test_matmul_of_whole_numbers_is_exact():
    # small whole numbers: every partial sum is exact in f32, whatever the order; a wrong k pairing or scale shows at once
    rng = np.random.default_rng(9)
    for M, N, K in ((16, 48, 640), (200, 140, 1300), (260, 300, 256)):
        a, b = rng.integers(-8, 9, size=(M, K)).astype(float), rng.integers(-8, 9, size=(N, K)).astype(float)
        a[:, ::7] *= 16                                              # other scales in other blocks and rows
        a[::3] *= 2
        pa, pb = binding.rl_f8_pack(rows(a, torch.float32)), binding.rl_f8_pack(rows(b, torch.float32))
        va, vb = f64(binding.rl_f8_unpack(pa, torch.float32)), f64(binding.rl_f8_unpack(pb, torch.float32))
        assert np.array_equal(f64(binding.rl_f8_matmul(pa, pb, torch.float32)), va @ vb.T)


def test_matmul_scales_apply_block_by_block():
    # one block of one row far larger than the rest, and one far smaller: 2^40 apart
    for M in (8, 40, 300):
        a = np.ones((M, 640))
        a[1, 128:256] *= 2.0 ** 40
        a[2, 512:] *= 2.0 ** -40
        b = np.zeros((70, 640))
        b[np.arange(70), np.arange(70) * 9 % 640] = 1.0
        b[5] *= 2.0 ** 30
        pa, pb = binding.rl_f8_pack(rows(a, torch.float32)), binding.rl_f8_pack(rows(b, torch.float32))
        assert np.array_equal(f64(binding.rl_f8_matmul(pa, pb, torch.float32)), a @ b.T)
        assert np.array_equal(f64(binding.rl_f8_matmul(pa, pb, torch.bfloat16)), a @ b.T)


@pytest.mark.parametrize("fa, fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2")])
def test_matmul_of_single_products_is_exact(fa, fb):
    # one value other than zero in each row of the second operand: every output is one product, of seven significant bits at most: exact in bf16 too
    rng = np.random.default_rng(8)
    for M, N, K in ((3, 40, 700), (50, 300, 517), (520, 600, 640), (1024, 513, 384)):
        a = rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, K)))
        b = np.zeros((N, K))
        b[np.arange(N), rng.integers(0, K, size=N)] = rng.choice([-1.0, 2.0, 0.5, 8.0], size=N)
        pa, pb = binding.rl_f8_pack(rows(a, torch.float32), fa), binding.rl_f8_pack(rows(b, torch.float32), fb)
        want = f64(binding.rl_f8_unpack(pa, torch.float32)) @ f64(binding.rl_f8_unpack(pb, torch.float32)).T
        for t in (torch.float32, torch.bfloat16):
            assert np.array_equal(f64(binding.rl_f8_matmul(pa, pb, t)), want)


@pytest.mark.parametrize("M, N, K", [(4096, 4096, 100), (4000, 4200, 384), (3900, 4099, 640), (8200, 2310, 1157)])
@pytest.mark.parametrize("fa, fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
def test_matmul_of_many_tiles(M, N, K, fa, fb):
    # 1, 3, 5 and 10 blocks of k; single products first, exact whatever the path; then sums, within the tolerance of the 8-bit matrix unit
    rng = np.random.default_rng(K)
    a = rng.normal(size=(M, K)) * 2.0 ** rng.integers(-9, 9, size=(M, 1))
    b = np.zeros((N, K))
    b[np.arange(N), rng.integers(0, K, size=N)] = rng.choice([-1.0, 2.0, 0.5, 8.0], size=N)
    pa, pb = binding.rl_f8_pack(rows(a, torch.float32), fa), binding.rl_f8_pack(rows(b, torch.float32), fb)
    va = f64(binding.rl_f8_unpack(pa, torch.float32))
    want = va[:, np.abs(b).argmax(1)] * b[np.arange(N), np.abs(b).argmax(1)]
    assert np.array_equal(f64(binding.rl_f8_matmul(pa, pb)), want)
    pb = binding.rl_f8_pack(rows(rng.normal(size=(N, K)) / K ** 0.5, torch.float32), fb)
    vb = f64(binding.rl_f8_unpack(pb, torch.float32))
    y = binding.rl_f8_matmul(pa, pb)
    for r in (slice(0, 40), slice(M // 2, M // 2 + 40), slice(M - 40, M)):
        want = va[r] @ vb.T
        tol = (2 * (K + 32) * U + CUT["bf16"]) * (np.abs(va[r]) @ np.abs(vb).T) + half_step(torch.bfloat16, want)
        assert np.all(np.abs(f64(y[r]) - want) <= tol)
        assert np.linalg.norm(f64(y[r]) - want) <= 2.0 ** -8 * np.linalg.norm(want)
    assert torch.equal(y, binding.rl_f8_matmul(pa, pb))


def test_matmul_keeps_what_is_not_finite_in_its_row():
    rng = np.random.default_rng(2)
    for M in (9, 33, 300):
        a = rng.normal(size=(M, 300))
        a[4, 299], a[6, 0] = np.nan, np.inf
        b = rng.normal(size=(80, 300))
        y = f64(binding.rl_f8_matmul(binding.rl_f8_pack(rows(a, torch.float32)), binding.rl_f8_pack(rows(b, torch.float32)), torch.float32))
        bad = np.zeros(M, bool)
        bad[[4, 6]] = True
        assert np.array_equal(np.isnan(y).all(1), bad) and np.isfinite(y[~bad]).all()


@pytest.mark.parametrize("M, N, K", [(1, 5, 40), (9, 300, 130), (300, 1157, 259), (2100, 512, 256)])
@pytest.mark.parametrize("dtype, fmt", [("bf16", "e4m3"), ("bf16", "e5m2"), ("f32", "e4m3")])
def test_weight_gradient_of_rows_without_a_gradient(M, N, K, dtype, fmt):
    """dy zero where x is infinite or no number: dW is that with such rows of x zero."""
    rng = np.random.default_rng(M + N)
    x, dy = rng.normal(size=(M, K)), rng.normal(size=(M, N))
    bad = rng.random(M) < 0.3
    bad[-1] = True
    dy[bad] = 0
    clean = x.copy()
    clean[bad] = 0
    x[bad, rng.integers(0, K, size=bad.sum())] = rng.choice([np.inf, -np.inf, np.nan], size=bad.sum())
    w = binding.rl_f8_pack_weight(rows(rng.normal(size=(N, K)), torch.float32))
    got = [binding.rl_f8_linear_backward(rows(dy, DT[dtype]), binding.rl_f8_pack(rows(v, DT[dtype]), fmt), w)[1] for v in (x, clean)]
    assert torch.isfinite(got[0]).all() and torch.equal(*got)
    dy[-1, N - 1] = 1                                                # with one value of dy it does count
    dw = binding.rl_f8_linear_backward(rows(dy, DT[dtype]), binding.rl_f8_pack(rows(x, DT[dtype]), fmt), w)[1]
    assert not torch.isfinite(dw[N - 1]).all()


def test_matmul_keeps_infinities_of_e5m2():
    rng = np.random.default_rng(12)
    for M in (9, 33, 300):
        a = rng.normal(size=(M, 300))
        a[4, 299], a[6, 0] = -np.inf, np.inf
        b = rng.choice([-1.0, 1.0], size=(80, 300)) * rng.uniform(0.5, 2, size=(80, 300))
        pa, pb = binding.rl_f8_pack(rows(a, torch.float32), "e5m2"), binding.rl_f8_pack(rows(b, torch.float32))
        for t in (torch.float32, torch.bfloat16):
            y = f64(binding.rl_f8_matmul(pa, pb, t))
            assert np.array_equal(y[6], np.inf * np.sign(b[:, 0])) and np.array_equal(y[4], -np.inf * np.sign(b[:, 299]))
            y[[4, 6]] = 0
            assert np.isfinite(y).all()


def test_matmul_at_the_ends_of_the_scales():
    # single products of powers of two, the factors near the ends of the scale bytes' range, the product inside f32's
    for M in (5, 40, 300):
        a, b = np.zeros((M, 256)), np.zeros((64, 256))
        a[:, 3], b[:, 3] = 2.0 ** -120, 2.0 ** 110
        a[1, 3], b[1, 3] = 2.0 ** -126, 2.0 ** 126
        a[:, 200], b[::2, 3] = 0, 0
        b[::2, 200] = 2.0 ** -118
        a[2, 200] = 2.0 ** 100
        pa, pb = binding.rl_f8_pack(rows(a, torch.float32)), binding.rl_f8_pack(rows(b, torch.float32))
        for t in (torch.float32, torch.bfloat16):
            assert np.array_equal(f64(binding.rl_f8_matmul(pa, pb, t)), a @ b.T), (M, t)


# ------------------------------------------------------------------ the linear layer
LINEAR = [(1, 1, 1), (1, 100, 300), (3, 17, 129), (16, 40, 256), (17, 40, 256), (127, 72, 130), (128, 64, 128), (129, 1157, 70), (300, 130, 517), (700, 264, 264), (1300, 300, 515)]


@pytest.mark.parametrize("M, N, K", LINEAR)
@pytest.mark.parametrize("dtype, fmt, gfmt, pad", [("bf16", "e4m3", "e5m2", 0), ("bf16", "e5m2", "e4m3", 3), ("f32", "e4m3", "e5m2", 0), ("f32", "e4m3", "e4m3", 1), ("bf16", "e4m3", "e4m3", 8)])
def test_linear(M, N, K, dtype, fmt, gfmt, pad):
    rng = np.random.default_rng(M * 3 + N + K)
    t = DT[dtype]
    x = rows(state(rng, M, K), t, pad)
    dy = rows(rng.normal(size=(M, N)) * (rng.random((M, 1)) < 0.8) * 1e-3, t, pad)
    w = binding.rl_f8_pack_weight(rows(rng.normal(size=(N, K)) / K ** 0.5, torch.float32))
    vw = f64(binding.rl_f8_unpack(w.rows, torch.float32))
    y, kept = binding.rl_f8_linear_forward(x, w, fmt)
    packed = binding.rl_f8_pack(x, fmt)
    assert torch.equal(kept.codes, packed.codes) and torch.equal(kept.scales, packed.scales)
    vx = f64(binding.rl_f8_unpack(kept, torch.float32))
    want = vx @ vw.T
    tol = (2 * (K + 32) * U + CUT[dtype]) * (np.abs(vx) @ np.abs(vw).T) + half_step(t, want)
    assert np.all(np.abs(f64(y) - want) <= tol)
    y2, none = binding.rl_f8_linear_forward(x, w, fmt, keep=False)
    assert torch.equal(y, y2) and none is None
    # backward
    dx, dw = binding.rl_f8_linear_backward(dy, kept, w, gfmt)
    vg = f64(binding.rl_f8_unpack(binding.rl_f8_pack(dy, gfmt), torch.float32))
    want = vg @ vw
    tol = (2 * (N + 32) * U + CUT[dtype]) * (np.abs(vg) @ np.abs(vw)) + half_step(t, want)
    assert np.all(np.abs(f64(dx) - want) <= tol)
    d = f64(dy)
    want = d.T @ vx
    mag = np.abs(d).T @ np.abs(vx)
    tol = 2 * (M + 32) * U * mag * (3 if dtype == "f32" else 1) + 1e-38
    assert np.all(np.abs(f64(dw) - want) <= tol), np.max(np.abs(f64(dw) - want) / tol)
    # one of the two alone; added to what is there
    only, none = binding.rl_f8_linear_backward(dy, None, w, gfmt, want_dw=False)
    assert torch.equal(only, dx) and none is None
    base = rng.normal(size=(N, K))
    into = rows(base, torch.float32, pad=2)
    none, got = binding.rl_f8_linear_backward(dy, kept, w, gfmt, want_dx=False, dw=into)
    assert none is None and got.data_ptr() == into.data_ptr()
    start = base.astype(np.float32).astype(np.float64)
    tol = tol + 4 * U * (np.abs(start) + mag)
    assert np.all(np.abs(f64(got) - start - want) <= tol)
    assert torch.all(into._base[:, K:] == 7)


def test_linear_without_rows():
    w = binding.rl_f8_pack_weight(torch.randn(20, 30, device="cuda"))
    x, dy = torch.empty(0, 30, device="cuda"), torch.empty(0, 20, device="cuda")
    y, kept = binding.rl_f8_linear_forward(x, w)
    dx, dw = binding.rl_f8_linear_backward(dy, kept, w)
    assert y.shape == (0, 20) and dx.shape == (0, 30) and torch.all(dw == 0)
    into = torch.ones(20, 30, device="cuda")
    binding.rl_f8_linear_backward(dy, kept, w, dw=into)
    assert torch.all(into == 1)


def test_f32_weight_gradient_is_exact_to_f32():
    # dy of 24 significant bits against powers of two: one product an entry, so that what is lost of dy shows
    rng = np.random.default_rng(4)
    M, N, K = 40, 24, 40
    x = np.zeros((M, K))
    x[np.arange(M), np.arange(M) % K] = 2.0 ** rng.integers(-5, 5, size=M)
    dy = rng.normal(size=(M, N)).astype(np.float32).astype(np.float64) * 10.0 ** rng.integers(-12, 12, size=(M, 1))
    w = binding.rl_f8_pack_weight(torch.randn(N, K, device="cuda"))
    t = rows(dy, torch.float32)
    _, dw = binding.rl_f8_linear_backward(t, binding.rl_f8_pack(rows(x, torch.float32)), w, want_dx=False)
    want = f64(t).T @ x
    assert np.all(np.abs(f64(dw) - want) <= 2 * U * np.abs(want))


# ------------------------------------------------------------------ streams, graphs
def _step(x, dy, gamma, beta, w):
    y, stats, kept = binding.rl_layer_norm_forward(x, gamma, beta, checkpoint="e4m3")
    z, zk = binding.rl_f8_linear_forward(y, w)
    dyn, dw = binding.rl_f8_linear_backward(dy, zk, w)
    dx, dg, db = binding.rl_layer_norm_backward(dyn, kept, stats, gamma)
    return y, z, dw, dx, dg, db


def _step_inputs(seed, M=700, K=640, N=520):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return n(M, K).bfloat16(), (n(M, N) * 1e-3).bfloat16(), n(K), n(K), binding.rl_f8_pack_weight(n(N, K) / K ** 0.5)


def test_another_stream_than_the_default():
    want = _step(*_step_inputs(1))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        args = _step_inputs(1)                                       # made on that stream as well, no wait in between
        got = _step(*args)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_a_captured_step_replays_with_new_inputs():
    args = _step_inputs(1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _step(*args)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(*args)
    for seed in (2, 3, 4):
        new = _step_inputs(seed)
        for a, b in zip(args[:4], new[:4]):
            a.copy_(b)
        for a, b in ((args[4].rows, new[4].rows), (args[4].cols, new[4].cols)):
            a.codes.copy_(b.codes)
            a.scales.copy_(b.scales)
        want = _step(*new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), seed


def test_offsets_past_32_bits():
    """The last rows of matrices of more than 2^32 bytes (codes: 2^31): what a call of those rows alone gives.  Small integers, whose sums are exact in any order."""
    R, H, N, last = 520_000, 4200, 70, 100
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randint(-4, 5, (R, H), generator=g, device="cuda", dtype=torch.int8).to(torch.bfloat16)
    gamma = torch.randn(H, generator=g, device="cuda")
    w = binding.rl_f8_pack_weight(torch.randint(-2, 3, (N, H), generator=g, device="cuda").to(torch.bfloat16))
    y, stats, kept = binding.rl_layer_norm_forward(x, gamma, checkpoint="e4m3")
    ys, ss, ks = binding.rl_layer_norm_forward(x[-last:], gamma, checkpoint="e4m3")
    assert torch.equal(y[-last:], ys) and torch.equal(stats[-last:], ss) and torch.equal(kept.codes[-last:], ks.codes) and torch.equal(kept.scales[-last:], ks.scales)
    for v, k, small in ((x, None, x[-last:]), (x, kept, ks)):
        dx = binding.rl_layer_norm_backward(y, k or v, stats, gamma)[0]
        assert torch.equal(dx[-last:], binding.rl_layer_norm_backward(ys, small, ss, gamma)[0])
        del dx
    del y
    assert torch.equal(binding.rl_f8_unpack(kept)[-last:], x[-last:])
    out, kept = binding.rl_f8_linear_forward(x, w)
    want, ks = binding.rl_f8_linear_forward(x[-last:], w)
    assert torch.equal(out[-last:], want) and torch.equal(kept.codes[-last:], ks.codes)
    dy = torch.zeros(R, N, device="cuda", dtype=torch.bfloat16)
    dy[-last:] = torch.randint(-2, 3, (last, N), generator=g, device="cuda").to(torch.bfloat16)
    dx, dw = binding.rl_f8_linear_backward(dy, kept, w)
    dxs, dws = binding.rl_f8_linear_backward(dy[-last:], ks, w)
    assert torch.equal(dx[-last:], dxs) and torch.equal(dw, dws) and torch.all(dx[:1000] == 0)
