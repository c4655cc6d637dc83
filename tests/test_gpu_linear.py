"""fs_linear_device against the definition in 64 bits.

Tolerance of an output: products of bf16 values are exact in fp32, products and
additions of the sum are otherwise off by at most one step of 2^-24 of a partial
sum that is at most `size` (the sum of all magnitudes).  Their signs are
independent, so 160 steps cover K <= 25088 additions (sqrt(25088) = 158 standard
deviations of a whole step), and 2 K steps the short sums; 8 more are the
epilogue's.  An activation stretches this by at most 1.13 and adds its own
evaluation, 16 steps of its argument; rounding to the output's type adds half a
step of the value."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2003_01538_amd import flexserve as fsb
from tests.device_rows import MARK, Rows, dtype_of, stream

pytestmark = pytest.mark.gpu
BF, F = fsb.FS_BF16, fsb.FS_F32
U = 2.0 ** -24


def tolerance(y, size, K, out):
    # values in [1, 2) lie 2^-7 (bf16, 8 significant bits) or 2^-23 (fp32, 24) apart: half a step is at most 2^-8 or 2^-24 of the value
    half = 2.0 ** -8 if out == BF else U
    return 1.13 * (min(2 * K, 160) + 24) * U * size + half * np.abs(y) + 1e-37


def make(M, N, K, prec, out, res, pads=(0, 0, 0, 0), leads=(0, 0, 0, 0), seed=0, bias=True):
    g = torch.Generator(device="cuda").manual_seed(seed + 31 * M + 7 * N + K)
    rnd = lambda r, c: torch.randn(r, c, device="cuda", generator=g)
    x = Rows(M, K, dtype_of(prec), pads[0], leads[0], rnd(M, K))
    w = Rows(N, K, dtype_of(prec), pads[1], leads[1], rnd(N, K) * (2.0 / max(K, 1)) ** 0.5)
    y = Rows(M, N, dtype_of(out), pads[2], leads[2])
    r = Rows(M, N, dtype_of(out), pads[3], leads[3], rnd(M, N)) if res else None
    b = torch.randn(N, device="cuda", generator=g) if bias else None
    return x, w, b, r, y


def call(x, w, b, r, y, prec, out, act, first, ldres=None, st=None):
    fsb.fs_linear_device(x.ptr, x.ld, w.ptr, w.ld, 0 if b is None else b.data_ptr(), 0 if r is None else r.ptr,
                         0 if r is None else (r.ld if ldres is None else ldres), y.ptr, y.ld, x.rows, w.rows, x.cols, prec,
                         out, act, first, stream() if st is None else st)


def check(x, w, b, r, y, out, act, first, res=None):
    rn = r.numpy() if r is not None and res is None else res
    want, size = ref.linear(x.numpy(), w.numpy(), None if b is None else b.cpu().numpy(), rn, act, first)
    got = y.numpy().astype(np.float64)
    off = np.abs(got - want) - tolerance(want, size, x.cols, out)
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))
    assert y.untouched()


@pytest.mark.parametrize("prec,out", [(BF, BF), (BF, F), (F, F)])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 1), (1, 1000, 512), (1, 17, 8), (2, 33, 40), (3, 10, 32), (5, 1000, 2048), (7, 100, 777), (16, 64, 64),
    (17, 65, 72), (31, 130, 250), (32, 1000, 512), (33, 256, 1024), (64, 512, 512), (65, 129, 65), (100, 96, 4100),
    (127, 127, 127), (128, 128, 128), (129, 257, 136), (255, 513, 64), (300, 40, 320), (513, 258, 192),
])
def test_sizes(gpu_lib, M, N, K, prec, out):
    x, w, b, r, y = make(M, N, K, prec, out, True)
    call(x, w, b, r, y, prec, out, 0, 0)
    check(x, w, b, r, y, out, 0, 0)


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("M,N,K", [(17, 100, 4096), (32, 1000, 2048), (31, 16, 25088), (20, 33, 1032), (25, 48, 520), (32, 65, 8200)])
def test_few_rows_over_a_long_reduction(gpu_lib, M, N, K, prec):
    x, w, b, r, y = make(M, N, K, prec, prec, True, pads=(0, 8, 0, 0), seed=10)
    call(x, w, b, r, y, prec, prec, 3, 0)
    check(x, w, b, r, y, prec, 3, 0)


@pytest.mark.parametrize("prec,out", [(BF, BF), (BF, F), (F, F)])
@pytest.mark.parametrize("act", [0, 1, 2, 3])
@pytest.mark.parametrize("res,first", [(0, 0), (1, 0), (1, 1)])
@pytest.mark.parametrize("M,N,K", [(4, 72, 96), (150, 200, 128), (40, 77, 33), (50, 72, 96)])
def test_epilogues(gpu_lib, M, N, K, prec, out, act, res, first):
    x, w, b, r, y = make(M, N, K, prec, out, res, seed=1)
    call(x, w, b, r, y, prec, out, act, first)
    check(x, w, b, r, y, out, act, first)


@pytest.mark.parametrize("prec,out", [(BF, BF), (F, F)])
@pytest.mark.parametrize("pads,leads", [
    ((8, 0, 0, 0), (0, 0, 0, 0)), ((0, 8, 8, 8), (8, 8, 8, 8)), ((1, 0, 0, 0), (0, 0, 0, 0)),
    ((0, 3, 0, 0), (0, 0, 0, 0)), ((0, 0, 5, 1), (0, 0, 0, 0)), ((0, 0, 0, 0), (1, 0, 0, 0)),
    ((0, 0, 0, 0), (0, 3, 0, 0)), ((0, 0, 0, 0), (0, 0, 1, 3)), ((4, 4, 4, 4), (4, 4, 4, 4)), ((2, 2, 2, 2), (2, 2, 2, 2)),
])
@pytest.mark.parametrize("M,N,K", [(3, 40, 128), (70, 136, 256), (260, 264, 128)])
def test_strides_and_alignment(gpu_lib, M, N, K, prec, out, pads, leads):
    x, w, b, r, y = make(M, N, K, prec, out, True, pads, leads, seed=2)
    call(x, w, b, r, y, prec, out, 1, 1)
    check(x, w, b, r, y, out, 1, 1)


@pytest.mark.parametrize("M", [2, 130])
def test_no_bias_one_residual_row_and_in_place(gpu_lib, M):
    x, w, b, r, y = make(M, 96, 64, BF, BF, True, bias=False, seed=3)
    call(x, w, None, None, y, BF, BF, 0, 0)
    check(x, w, None, None, y, BF, 0, 0)
    call(x, w, None, r, y, BF, BF, 2, 0, ldres=0)  # the first row of r for every row of y
    check(x, w, None, r, y, BF, 2, 0, res=np.broadcast_to(r.numpy()[:1], (M, 96)))
    before = r.numpy().copy()
    call(x, w, None, r, r, BF, BF, 0, 0)
    check(x, w, None, r, r, BF, 0, 0, res=before)


@pytest.mark.parametrize("prec,out", [(BF, BF), (F, F)])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("M,N,K", [
    (4000, 4090, 520), (4000, 4090, 2056), (2000, 4090, 2056), (1000, 4090, 2056), (1000, 4090, 520), (500, 4090, 520), (4096, 4096, 64),
    (514, 1061, 128), (135, 2834, 2264), (509, 1679, 2916), (486, 2707, 40),
])
def test_many_tiles(gpu_lib, M, N, K, pad, prec, out):
    # the tiles of 64 x 32 up to 256 x 256, most with ragged edges; the definition in 64 bits on the GPU
    x, w, b, r, y = make(M, N, K, prec, out, True, pads=(pad, pad, pad, pad), seed=9)
    call(x, w, b, r, y, prec, out, 1, 1)
    xd, wd, rd = x.view.double(), w.view.double(), r.view.double()
    want = (xd @ wd.t() + b.double() + rd).clamp_min(0)
    size = xd.abs() @ wd.abs().t() + b.double().abs() + rd.abs()
    half = 2.0 ** -8 if out == BF else U  # as in tolerance()
    off = (y.view.double() - want).abs() - (1.13 * (min(2 * K, 160) + 24) * U * size + half * want.abs() + 1e-37)
    assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()) // N, int(off.argmax()) % N)
    assert y.untouched()


@pytest.mark.parametrize("M,N,K", [(20, 64, 512), (600, 1024, 64), (4096, 4096, 64)])
def test_one_residual_row_and_in_place_on_every_kind_of_tile(gpu_lib, M, N, K):
    x, w, b, r, y = make(M, N, K, BF, BF, True, seed=11)
    product = x.view.double() @ w.view.double().t()
    size = x.view.double().abs() @ w.view.double().abs().t()

    def near(res, got):
        want = product + res
        off = (got.double() - want).abs() - (1.13 * (min(2 * K, 160) + 24) * U * (size + res.abs()) + 2.0 ** -8 * want.abs())  # as in tolerance()
        assert bool((off <= 0).all()), float(off.max())

    call(x, w, None, r, y, BF, BF, 0, 1, ldres=0)
    near(r.view[:1].double(), y.view)
    before = r.view.double().clone()
    call(x, w, None, r, r, BF, BF, 0, 0)
    near(before, r.view)
    assert r.untouched()


@pytest.mark.parametrize("M", [1, 70, 3000])
def test_empty_sum_and_no_rows(gpu_lib, M):
    x, w, b, r, y = make(M, 50, 0, BF, F, True, seed=4)
    fsb.fs_linear_device(0, 0, 0, 0, b.data_ptr(), r.ptr, r.ld, y.ptr, y.ld, M, 50, 0, BF, F, 3, 1, stream())
    check(x, w, b, r, y, F, 3, 1)
    y2 = Rows(M, 50, torch.float32)
    fsb.fs_linear_device(x.ptr, 0, w.ptr, 0, 0, 0, 0, y2.ptr, 50, 0, 50, 0, BF, F, 0, 0, stream())
    assert (y2.numpy() == MARK).all()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("M,N,K", [(2, 40, 72), (140, 130, 200), (140, 130, 72)])
def test_not_finite_values_stay_in_their_rows(gpu_lib, M, N, K, prec):
    # one NaN in x's row 1, one inf in w's row 2: only y's row 1 and column 2 see them, and
    # what lies beside the rows (NaN here) is not read into any sum
    x, w, b, r, y = make(M, N, K, prec, F, False, pads=(8, 8, 0, 0), seed=5)
    for t in (x, w):
        keep = t.view.clone()
        t.buf.fill_(float("nan"))
        t.view.copy_(keep)
    x.view[1, K - 1] = float("nan")
    w.view[2, 0] = float("inf")
    call(x, w, b, None, y, prec, F, 0, 0)
    got = y.numpy()
    assert np.isnan(got[1]).all() and not np.isfinite(got[:, 2]).any()
    fine = np.ones((M, N), bool)
    fine[1] = False
    fine[:, 2] = False
    with np.errstate(invalid="ignore"):
        want, size = ref.linear(x.numpy(), w.numpy(), b.cpu().numpy())
    assert (np.abs(got[fine] - want[fine]) <= tolerance(want, size, K, F)[fine]).all()


def test_activations_at_their_ends(gpu_lib):
    # s = +-large, 0 and inf through the bias; K = 0
    b = torch.tensor([-3.4e38, -200.0, -90.0, -20.0, -0.0, 0.0, 20.0, 90.0, 200.0, 3.4e38, float("inf")], device="cuda")
    for act in range(4):
        y = Rows(1, 11, torch.float32)
        fsb.fs_linear_device(0, 0, 0, 0, b.data_ptr(), 0, 0, y.ptr, 11, 1, 11, 0, F, F, act, 0, stream())
        with np.errstate(over="ignore", invalid="ignore"):
            want = ref.activation(b.cpu().numpy().astype(np.float64), act)
        got = y.numpy()[0].astype(np.float64)
        ok = np.isfinite(want)
        assert (np.abs(got[ok] - want[ok]) <= 32 * U * np.abs(want[ok]) + 1e-6).all(), (act, got, want)
        assert got[-1] == np.inf


def test_other_stream_and_two_calls_at_once(gpu_lib):
    a, c = torch.cuda.Stream(), torch.cuda.Stream()
    one, two = make(40, 1000, 2048, BF, BF, True, seed=6), make(300, 512, 512, BF, BF, True, seed=7)
    torch.cuda.synchronize()
    for _ in range(10):
        call(*one, BF, BF, 2, 0, st=a.cuda_stream)
        call(*two, BF, BF, 2, 0, st=c.cuda_stream)
    torch.cuda.synchronize()
    check(*one, BF, 2, 0)
    check(*two, BF, 2, 0)


@pytest.mark.parametrize("M", [1, 200])
def test_captured_and_replayed(gpu_lib, M):
    x, w, b, r, y = make(M, 520, 1024, BF, BF, True, seed=8)
    call(x, w, b, r, y, BF, BF, 1, 1)
    torch.cuda.synchronize()
    want = y.view.clone()
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        call(x, w, b, r, y, BF, BF, 1, 1, st=s.cuda_stream)
    for i in range(4):
        y.view.fill_(MARK)
        x.view.copy_(x.view.roll(1, 1) if i % 2 else x.view)
        call(x, w, b, r, y, BF, BF, 1, 1)
        want = y.view.clone()
        y.view.fill_(MARK)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.view, want), i


def test_host_memory_is_refused(gpu_lib):
    x, w, b, r, y = make(2, 8, 8, BF, F, False)
    host = torch.zeros(64)
    with pytest.raises(fsb.FsError) as e:
        fsb.fs_linear_device(host.data_ptr(), 8, w.ptr, 8, 0, 0, 0, y.ptr, 8, 2, 8, 8, BF, F, 0, 0, stream())
    assert e.value.status == fsb.FS_ERR_INVALID and "device memory" in str(e.value)
    call(x, w, b, r, y, BF, F, 0, 0)  # and the next call is fine
    check(x, w, b, r, y, F, 0, 0)


def test_rows_beyond_32_bit_offsets(gpu_lib):
    # rows 2^22 elements apart: the last of 600 rows starts 2.5e9 elements into the buffer
    far = (1 << 22) + 8
    for M, N in ((600, 24), (24, 600)):
        x = torch.randn(M, 64, device="cuda").bfloat16()
        w = torch.randn(N, 64, device="cuda").bfloat16()
        big = torch.empty(600 * far, dtype=torch.bfloat16, device="cuda")
        v = big.view(600, far)[:, :64]
        v.copy_(x if M == 600 else w)
        y = Rows(M, N, torch.float32)
        px, lx, pw, lw = ((v.data_ptr(), far, w.data_ptr(), 64) if M == 600 else (x.data_ptr(), 64, v.data_ptr(), far))
        fsb.fs_linear_device(px, lx, pw, lw, 0, 0, 0, y.ptr, y.ld, M, N, 64, BF, F, 0, 0, stream())
        want, size = ref.linear(x.float().cpu().numpy(), w.float().cpu().numpy())
        assert (np.abs(y.numpy() - want) <= tolerance(want, size, 64, F)).all()
        del big, v


@pytest.mark.parametrize("M,N", [(1, 1 << 26), (12, (1 << 24) + 5), (1 << 26, 65)])
def test_more_outputs_than_a_launch_has_threads(gpu_lib, M, N):
    # one product per output: exact in fp32, rounded once
    x, w, b, r, y = make(M, N, 1, BF, BF, M <= 12, seed=12)
    call(x, w, b, r, y, BF, BF, 0, 0)
    for m in range(0, M, 1 << 24):
        rows = slice(m, m + (1 << 24))
        want = x.view[rows].float() * w.view.float().t() + b
        assert torch.equal(y.view[rows], (want if r is None else want + r.view.float()).bfloat16()), m
    assert bool((y.buf[-64:] == MARK).all())


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 0), (0, 1), (3, 2), (2, 1), (8, 0)])
@pytest.mark.parametrize("M,N,K", [(9, 20, 900), (41, 58, 2049), (70, 130, 4100), (120, 339, 1001), (300, 300, 263), (12, 40, 9)])
def test_rows_between_two_words_in_small_tiles(gpu_lib, M, N, K, pad, lead, prec):
    x, w, b, r, y = make(M, N, K, prec, prec, True, pads=(pad, pad, 0, 0), leads=(lead, lead, 0, 0), seed=13)
    for t in (x, w):  # what lies beside the rows is read into no sum
        keep = t.view.clone()
        t.buf.fill_(float("nan"))
        t.view.copy_(keep)
    call(x, w, b, r, y, prec, prec, 0, 0)
    check(x, w, b, r, y, prec, 0, 0)


@pytest.mark.parametrize("act", [2, 3])
@pytest.mark.parametrize("out", [BF, F])
@pytest.mark.parametrize("M", [1, 300])
def test_the_tails_of_the_activations(gpu_lib, M, out, act):
    # s alone through the bias (K = 0), so that nothing but the activation rounds.  GELU for fp32: the
    # fit 2 steps of U, the reciprocal and its argument 3, the polynomial 4, the exponential with
    # its correction 3, three products 3; SiLU fewer: 16 for both.  For bf16 the exponent's own roundings
    # stay, three steps of it; half a step of the value comes last.  Exponentials below 2^-126 may be 0.
    from scipy.special import log_ndtr
    v = torch.cat([torch.arange(-13.0, 13.0, 1 / 64), torch.arange(-100.0, 100.0, 0.37)]).cuda()
    N = len(v)
    y = Rows(M, N, dtype_of(out))
    fsb.fs_linear_device(0, 0, 0, 0, v.data_ptr(), 0, 0, y.ptr, y.ld, M, N, 0, BF, out, act, 0, stream())
    s = v.cpu().numpy().astype(np.float64)
    with np.errstate(over="ignore"):
        want = s * np.exp(log_ndtr(s)) if act == 2 else s / (1 + np.exp(-s))
    exponent = np.minimum(np.abs(s), 13.2) ** 2 / 2 if act == 2 else np.minimum(np.abs(s), 88)
    steps = 16 * U if out == F else 16 * U + 3 * U * exponent + 2.0 ** -8
    off = np.abs(y.numpy().astype(np.float64) - want) - (steps * np.abs(want) + np.abs(s) * 2.0 ** -126)
    assert (off <= 0).all(), (off.max(), s[off.max(0).argmax()])


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("pad", [8, 3])
@pytest.mark.parametrize("M,N,K", [(1, 2048, 4096), (8, 2049, 4096), (1, 33, 16384), (5, 2100, 8192), (8, 2064, 16376), (3, 1, 8), (7, 2048, 24),
                                   (6, 5000, 4099), (1, 2049, 4095), (8, 16, 25087)])
def test_up_to_eight_rows_by_either_kernel(gpu_lib, M, N, K, pad, prec):
    x, w, b, r, y = make(M, N, K, prec, prec, True, pads=(pad, pad, 3, 1), seed=14)
    for t in (x, w):  # what lies beside the rows is read into no sum
        keep = t.view.clone()
        t.buf.fill_(float("nan"))
        t.view.copy_(keep)
    call(x, w, b, r, y, prec, prec, 2, 1)
    check(x, w, b, r, y, prec, 2, 1)


def against_64_bits_on_the_gpu(x, w, b, r, y, K, out):
    xd, wd, rd = x.view.double(), w.view.double(), r.view.double()
    want = xd @ wd.t() + b.double() + rd
    size = xd.abs() @ wd.abs().t() + b.double().abs() + rd.abs()
    half = 2.0 ** -8 if out == BF else U  # as in tolerance()
    off = (y.view.double() - want).abs() - (1.13 * (min(2 * K, 160) + 24) * U * size + half * want.abs() + 1e-37)
    assert bool((off <= 0).all()), (float(off.max()), int(off.argmax()) // y.cols, int(off.argmax()) % y.cols)
    assert y.untouched()


@pytest.mark.parametrize("pad,lead", [(0, 0), (3, 0), (8, 1)])
@pytest.mark.parametrize("M,N,K", [
    (45, 65, 2463), (9, 17, 31), (1398, 33, 100), (65, 1407, 68), (1347, 164, 100), (1345, 321, 68), (322, 1481, 260), (322, 1481, 257),
    (386, 1222, 5), (1475, 322, 68), (1154, 842, 36), (1346, 1060, 36), (1409, 1415, 68), (1000, 4090, 1030), (4200, 955, 2052),
    (2000, 4090, 520), (4000, 4090, 2056), (33, 64, 32), (64, 33, 96), (130, 97, 3), (51, 2061, 68), (2361, 195, 515), (99, 2362, 100),
    (2119, 33, 64), (257, 2242, 1000),
])
def test_every_tile_of_fp32(gpu_lib, M, N, K, pad, lead):
    # ragged edges, the reduction's last part, rows at any element; what lies beside the rows is read into no sum
    x, w, b, r, y = make(M, N, K, F, F, True, pads=(pad, pad, pad, 1), leads=(lead, lead, lead, 0), seed=15)
    for t in (x, w):
        keep = t.view.clone()
        t.buf.fill_(float("nan"))
        t.view.copy_(keep)
    call(x, w, b, r, y, F, F, 0, 1)
    against_64_bits_on_the_gpu(x, w, b, r, y, K, F)
    first = y.view.clone()
    call(x, w, b, r, y, F, F, 0, 1)
    assert torch.equal(y.view, first)
    call(x, w, b, r, r, F, F, 0, 1)  # over the residual
    assert torch.equal(r.view, first) and r.untouched()


@pytest.mark.parametrize("M,N,K", [(40, 70, 1000), (70, 1407, 260), (400, 1400, 100), (1154, 842, 37)])
def test_fp32_values_that_are_not_finite_stay_in_their_rows(gpu_lib, M, N, K):
    x, w, b, r, y = make(M, N, K, F, F, True, pads=(1, 3, 0, 0), seed=16)
    x.view[1, K - 1] = float("nan")
    w.view[2, 0] = float("inf")
    call(x, w, b, r, y, F, F, 0, 1)
    assert bool(y.view[1].isnan().all()) and not bool(y.view[:, 2].isfinite().any())
    x.view[1], w.view[2] = 0, 0
    y.view[1], y.view[:, 2] = b + r.view[1], b[2] + r.view[:, 2]
    against_64_bits_on_the_gpu(x, w, b, r, y, K, F)


def test_fp32_rows_that_are_far_apart(gpu_lib):
    # rows 2^22 elements apart: more than a tile's offsets reach, and beyond 2^31 bytes in all
    far = (1 << 22) + 1
    for M, N in ((150, 70), (70, 150), (5, 150), (150, 5)):
        x, w = torch.randn(M, 67, device="cuda"), torch.randn(N, 67, device="cuda")
        big = torch.empty(150 * far, device="cuda")
        v = big.view(150, far)[:, :67]
        v.copy_(x if M == 150 else w)
        y = Rows(M, N, torch.float32)
        px, lx, pw, lw = ((v.data_ptr(), far, w.data_ptr(), 67) if M == 150 else (x.data_ptr(), 67, v.data_ptr(), far))
        fsb.fs_linear_device(px, lx, pw, lw, 0, 0, 0, y.ptr, y.ld, M, N, 67, F, F, 0, 0, stream())
        want, size = ref.linear(x.cpu().numpy(), w.cpu().numpy())
        assert (np.abs(y.numpy() - want) <= tolerance(want, size, 67, F)).all()
        del big, v


@pytest.mark.parametrize("M,N", [(12, (1 << 24) + 5), ((1 << 26), 5)])
def test_more_fp32_outputs_than_a_launch_has_threads(gpu_lib, M, N):
    x, w, b, r, y = make(M, N, 1, F, F, False, seed=17)  # one product and one addition per output
    call(x, w, b, None, y, F, F, 0, 0)
    for m in range(0, M, 1 << 24):
        rows = slice(m, m + (1 << 24))
        want = (x.view[rows].double() * w.view.double().t() + b.double())
        off = (y.view[rows].double() - want).abs() - 2 * U * (want.abs() + b.double().abs())
        assert bool((off <= 0).all())
    assert bool((y.buf[-64:] == MARK).all())


@pytest.mark.parametrize("M,N,K", [(45, 65, 2463), (322, 1481, 260), (1409, 1415, 68)])
def test_fp32_tiles_captured_and_on_two_streams(gpu_lib, M, N, K):
    one, two = make(M, N, K, F, F, True, pads=(3, 3, 0, 0), seed=18), make(M, N, K, F, F, True, pads=(4, 4, 0, 0), seed=19)
    torch.cuda.synchronize()
    a, c = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        call(*one, F, F, 2, 0, st=a.cuda_stream)
        call(*two, F, F, 3, 1, st=c.cuda_stream)
    torch.cuda.synchronize()
    check(*one, F, 2, 0)
    check(*two, F, 3, 1)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        call(*one, F, F, 2, 0, st=s.cuda_stream)
        call(*two, F, F, 3, 1, st=s.cuda_stream)
    for i in range(3):
        want = []
        for t, act, first in ((one, 2, 0), (two, 3, 1)):
            t[0].view.copy_(t[0].view.roll(1, 1))
            call(*t, F, F, act, first)
            want.append(t[4].view.clone())
            t[4].view.fill_(MARK)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(one[4].view, want[0]) and torch.equal(two[4].view, want[1]), i
