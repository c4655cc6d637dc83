"""fs_distill_device and fs_distill_grad_device against the definition in 64
bits, and the gradient against differences of the loss.

Tolerances, in steps of U = 2^-24: q and p are quotients of an exponential by a
sum of them.  The argument of an exponential is off by two steps of itself and the
sum by some 32 of itself, so p and q are within (64 + 4 |ln p|) U of themselves
and ln p, ln q within (128 + 8 |ln p|) U.  A loss is an average (weights q) of
differences of the two; a gradient is their difference times weight / temperature
(three more steps), rounded to the logits' type: half a step of the value."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2003_01538_amd import flexserve as fsb
from tests.device_rows import Rows, dtype_of, stream

pytestmark = pytest.mark.gpu
BF, F = fsb.FS_BF16, fsb.FS_F32
U = 2.0 ** -24


class Call:
    def __init__(self, z, ids, u, prec, tau=1.0, weight=True, pad=0, lead=0, padg=0, split=True, in_place=False):
        R, C = z.shape
        self.z, self.prec, self.tau = Rows(R, C, dtype_of(prec), pad, lead, z), prec, tau
        self.ids, self.u, self.K = ids.to(device="cuda", dtype=torch.int32).contiguous(), u.float().cuda().contiguous(), ids.shape[1]
        g = torch.Generator(device="cuda").manual_seed(R + C)
        self.weight = torch.randn(R, device="cuda", generator=g) if weight else None
        self.loss, self.stats = Rows(R, 1, torch.float32), Rows(R, 2, torch.float32)
        self.student = self.z.numpy().copy()
        self.grad = self.z if in_place else Rows(R, C, dtype_of(prec), padg, lead)
        self.scratch = torch.empty(fsb.FS_ROW_SCRATCH_BYTES, dtype=torch.uint8, device="cuda") if split else None

    def head(self):
        z = self.z
        return (z.ptr, z.ld, z.rows, z.cols, self.prec, self.ids.data_ptr(), self.u.data_ptr(), self.K, self.tau,
                self.weight.data_ptr() if self.weight is not None else 0)

    def run(self, loss=True, grad=True, st=None):
        fsb.fs_distill_device(*self.head(), self.loss.ptr if loss else 0, self.stats.ptr if loss else 0,
                              self.grad.ptr if grad else 0, self.grad.ld, 0 if self.scratch is None else self.scratch.data_ptr(),
                              stream() if st is None else st)
        return self

    def run_grad(self, st=None):
        fsb.fs_distill_grad_device(*self.head(), self.stats.ptr, self.grad.ptr, self.grad.ld, stream() if st is None else st)
        return self

    def want(self):
        return ref.distill(self.student, self.ids.cpu().numpy(), self.u.cpu().numpy(), self.tau,
                           None if self.weight is None else self.weight.cpu().numpy())

    def check_loss(self):
        w, n = self.want(), self.student.shape[1]
        lp = ref.log_softmax(self.student, self.tau)
        big = np.zeros(len(lp))
        for r in range(len(lp)):
            at = [(w["q"][r, j], lp[r, c]) for j, c in enumerate(self.ids[r].tolist()) if 0 <= c < n and w["q"][r, j] > 0]
            big[r] = sum(q * (256 + 8 * abs(v) + 8 * abs(np.log(q))) for q, v in at if np.isfinite(v))
        near(self.loss.numpy()[:, 0], w["loss"], (big + 8) * U)
        st = self.stats.numpy()
        near(st[:, 1], w["stats"][:, 1], (128 + 8 * np.abs(np.nan_to_num(w["stats"][:, 1], posinf=0, neginf=0))) * U)
        clean = ~np.isnan(w["stats"][:, 0])
        assert np.array_equal(st[clean, 0], w["stats"][clean, 0])
        assert self.loss.untouched() and self.stats.untouched()
        return self

    def check_grad(self):
        w = self.want()
        with np.errstate(divide="ignore", invalid="ignore"):
            p_off = w["p"] * (64 + 4 * np.abs(np.where(w["p"] > 0, np.log(w["p"]), 0))) * U
            q_off = w["q"] * (64 + 4 * np.abs(np.where(w["q"] > 0, np.log(w["q"]), 0))) * U
        off = np.nan_to_num(p_off)
        for r, row in enumerate(self.ids.tolist()):
            for j, c in enumerate(row):
                if 0 <= c < off.shape[1]:
                    off[r, c] += np.nan_to_num(q_off[r, j])
        scale = np.abs(1.0 if self.weight is None else self.weight.cpu().numpy()) / self.tau
        # values in [1, 2) lie 2^-7 (bf16) or 2^-23 (fp32) apart: half a step is at most 2^-8 or 2^-24 of the value
        half = 2.0 ** -8 if self.prec == BF else U
        # an exponential below 2^-126, the least normal fp32 number, may be 0: times scale in the gradient
        least = 2.0 ** -126 * np.reshape(scale, (-1, 1) if np.ndim(scale) else (1, 1))
        tol = off * np.reshape(scale, (-1, 1) if np.ndim(scale) else (1, 1)) + (half + 3 * U) * np.abs(np.nan_to_num(w["grad"])) + least + 1e-37
        near(self.grad.numpy(), w["grad"], tol)
        assert self.grad.untouched()
        return self


def near(got, want, tol):
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = np.isfinite(want) & np.isfinite(got) & (np.abs(got.astype(np.float64) - want) <= tol)
    assert (same | ok).all(), (np.argwhere(~(same | ok))[:4], got[~(same | ok)][:4], want[~(same | ok)][:4])


def inputs(R, C, K, seed=0):
    g = torch.Generator(device="cuda").manual_seed(100 * seed + R + 3 * C + K)
    z = torch.randn(R, C, device="cuda", generator=g) * 3
    ids = torch.randint(0, C, (R, K), device="cuda", generator=g)  # a class may come twice
    return z, ids, torch.randn(R, K, device="cuda", generator=g) * 2


SIZES = [(1, 1, 1), (2, 2, 3), (3, 10, 5), (256, 1000, 5), (5, 63, 64), (4, 64, 128), (9, 1001, 8), (2, 4096, 32), (3, 4097, 128),
         (1, 20000, 20), (33, 16385, 4), (1, 131072, 64), (7, 100003, 16), (600, 257, 3), (2, 262144, 10), (300, 9001, 7),
         (6, 33000, 9), (5, 65536, 12), (4, 70000, 3)]


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("R,C,K", SIZES)
def test_sizes(gpu_lib, R, C, K, prec, split):
    c = Call(*inputs(R, C, K), prec, 2.0, split=split)
    c.run(grad=False).check_loss()
    c.run(loss=False).check_grad()
    c.grad.view.fill_(c.grad.mark())
    c.loss.view.fill_(c.loss.mark())
    c.run().check_loss().check_grad()
    c.grad.view.fill_(c.grad.mark())
    c.run_grad().check_grad()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("pad,lead,padg", [(0, 1, 0), (1, 0, 0), (0, 0, 3), (4, 4, 8), (8, 8, 8), (2, 6, 1), (7, 5, 7)])
@pytest.mark.parametrize("R,C", [(3, 50), (2, 5001), (1, 70000), (70, 1003)])
def test_strides_and_alignment(gpu_lib, R, C, pad, lead, padg, prec):
    c = Call(*inputs(R, C, 9), prec, pad=pad, lead=lead, padg=padg)
    c.run().check_loss().check_grad()
    c.grad.view.fill_(c.grad.mark())
    c.run_grad().check_grad()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("R,C", [(3, 50), (2, 5001), (1, 70000), (300, 1000), (4, 140000)])
def test_gradient_over_the_logits(gpu_lib, R, C, prec):
    z, ids, u = inputs(R, C, 9)
    Call(z, ids, u, prec, in_place=True, pad=2).run().check_loss().check_grad()
    c = Call(z, ids, u, prec, in_place=True)
    c.run(grad=False).run_grad().check_grad()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("tau", [1e-6, 0.05, 1.0, 30.0, 1e6])
def test_temperatures(gpu_lib, tau, prec):
    Call(*inputs(5, 1500, 6), prec, tau, weight=False).run().check_loss().check_grad()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("C", [20, 1000, 5000, 40000, 150000])
def test_rows_without_a_teacher_and_values_that_are_not_finite(gpu_lib, C, prec):
    inf, nan = float("inf"), float("nan")
    low = torch.finfo(dtype_of(prec)).min
    z, _, u = inputs(16, C, 4, seed=3)
    ids = torch.tensor([[0, 1, C - 1, C // 2]] * 16)
    ids[0] = -1                                   # no entry
    ids[1] = torch.tensor([C, C + 5, -7, 2 ** 31 - 1])
    u[2] = -inf                                   # no mass
    ids[3, 1:] = -1                               # one entry
    u[4, 2] = -inf
    ids[5] = 3                                    # one class four times
    ids[6, 1] = 0
    z[7] = -inf                                   # the student has nothing left
    z[8, 1] = -inf                                # ... not the class that the teacher wants
    z[9, torch.rand(C, device="cuda") < 0.9] = -inf
    z[9, [0, 1, C - 1, C // 2]] = 1.0
    z[10] = low
    z[11, C // 3] = nan
    z[12, C // 3] = inf
    z[13, C // 3] = nan
    ids[13] = -1                                  # not trained on: 0 whatever the logits are
    u[14] = torch.finfo(torch.float32).min
    u[15, 1] = nan
    for split in (True, False):
        c = Call(z, ids, u, prec, 0.7, split=split)
        c.run().check_loss().check_grad()
        c.grad.view.fill_(c.grad.mark())
        c.run_grad().check_grad()


@pytest.mark.parametrize("C", [300, 70000])
def test_gradient_against_differences(gpu_lib, C):
    # central differences of the loss at a few classes, the two losses in fp32: a step h of 0.25 makes
    # an error of h^2 / 6 times the third derivative (at most 1 / (6 sqrt 3) for a softmax) and 2 (256 + 8 * 12) U / (2 h) of rounding
    z, ids, u = inputs(1, C, 6, seed=4)
    z[0, :3] += 6.0
    c = Call(z, ids, u, F, weight=False).run()
    at = [0, 1, 2, int(ids[0, 0]), int(ids[0, 5]), C - 1]
    up = torch.cat([z + 0.25 * torch.eye(C, device="cuda")[i][None] if C < 1000 else z.index_add(1, torch.tensor([i], device="cuda"), torch.full((1, 1), 0.25, device="cuda")) for i in at])
    dn = torch.cat([z.index_add(1, torch.tensor([i], device="cuda"), torch.full((1, 1), -0.25, device="cuda")) for i in at])
    n = len(at)
    lu = Call(up, ids.expand(n, -1), u.expand(n, -1), F).run(grad=False).loss.numpy()[:, 0]
    ld = Call(dn, ids.expand(n, -1), u.expand(n, -1), F).run(grad=False).loss.numpy()[:, 0]
    g = c.grad.numpy()[0, at]
    assert np.abs(g - (lu - ld) / 0.5).max() <= 0.25 ** 2 / 6 / (6 * 3 ** 0.5) + 2 * (256 + 96) * U / 0.5


def test_rows_at_a_32_bit_offset(gpu_lib):
    C, R = 1 << 20, 2100
    big = torch.zeros(R * C, device="cuda").view(R, C)
    z, ids, u = inputs(2, C, 5, seed=5)
    big[R - 2:] = z
    ids = torch.cat([torch.zeros(R - 2, 5, device="cuda", dtype=torch.long), ids]).int()
    u = torch.cat([torch.zeros(R - 2, 5, device="cuda"), u])
    loss, stats = torch.empty(R, device="cuda"), torch.empty(R, 2, device="cuda")
    args = (big.data_ptr(), C, R, C, F, ids.data_ptr(), u.data_ptr(), 5, 1.0, 0)
    fsb.fs_distill_device(*args, loss.data_ptr(), stats.data_ptr(), big.data_ptr(), C, 0, stream())  # the gradient over the logits
    want = ref.distill(z.cpu().numpy(), ids[R - 2:].cpu().numpy(), u[R - 2:].cpu().numpy(), 1.0)
    assert np.abs(loss[R - 2:].cpu().numpy() - want["loss"]).max() <= (256 + 16 * 40) * U
    assert np.abs(big[R - 2:].cpu().numpy() - want["grad"]).max() <= 256 * U
    assert (big[: R - 2, 1:] == big[0, 1]).all() and abs(float(big[0, 1]) * C - 1) < 128 * U


@pytest.mark.parametrize("R,C", [(3, 900), (2, 5000), (3, 70000), (70, 70000)])
def test_outputs_that_are_not_asked_for(gpu_lib, R, C):
    c = Call(*inputs(R, C, 5, seed=9), F)
    c.run()
    loss, stats, grad = (torch.full_like(t.view, t.mark()) for t in (c.loss, c.stats, c.grad))
    sc = c.scratch.data_ptr()
    fsb.fs_distill_device(*c.head(), loss.data_ptr(), 0, 0, c.grad.ld, sc, stream())
    fsb.fs_distill_device(*c.head(), 0, stats.data_ptr(), 0, c.grad.ld, sc, stream())
    fsb.fs_distill_device(*c.head(), 0, 0, grad.data_ptr(), C, sc, stream())
    for got, want in ((loss, c.loss), (stats, c.stats), (grad, c.grad)):
        assert torch.equal(got, want.view)


def test_more_rows_than_workgroups(gpu_lib):
    R, C, K = (1 << 20) + 70, 5, 2
    z, _, u = inputs(R, C, K, seed=8)
    ids = torch.stack([torch.arange(R, device="cuda") % C, (torch.arange(R, device="cuda") + 2) % C], 1).int().contiguous()
    loss, stats, grad, again = (torch.empty(*s, device="cuda") for s in ((R,), (R, 2), (R, C), (R, C)))
    head = (z.data_ptr(), C, R, C, F, ids.data_ptr(), u.data_ptr(), K, 2.0, 0)
    fsb.fs_distill_device(*head, loss.data_ptr(), stats.data_ptr(), grad.data_ptr(), C, 0, stream())
    fsb.fs_distill_grad_device(*head, stats.data_ptr(), again.data_ptr(), C, stream())
    lp, q = torch.log_softmax(z.double() / 2, 1), torch.softmax(u.double() / 2, 1)
    want = (q * (q.log() - lp.gather(1, ids.long()))).sum(1)
    g = lp.exp().scatter_add(1, ids.long(), -q) / 2
    # |ln p|, |ln q| up to 20 here
    assert bool(((loss.double() - want).abs() <= (256 + 16 * 20) * U).all())
    for got in (grad, again):
        assert bool(((got.double() - g).abs() <= 2 * (64 + 4 * 20) * U / 2 + 4 * U * g.abs()).all())


def test_streams_and_graphs(gpu_lib):
    s = torch.cuda.Stream()
    calls = [Call(*inputs(R, C, 8, seed=6), F) for R, C in ((2, 130000), (96, 1000), (3, 40000))]
    for c in calls:
        c.scratch = calls[0].scratch
        c.run().run_grad()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for c in calls:
            c.run(st=s.cuda_stream)
    for i in range(4):
        for c in calls:
            c.z.view.copy_(c.z.view.roll(37, 1))
            c.student = c.z.numpy().copy()
            for t in (c.loss, c.stats, c.grad):
                t.view.fill_(t.mark())
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for c in calls:
            c.check_loss().check_grad()


def test_same_bits_every_time(gpu_lib):
    c = Call(*inputs(3, 131072, 64, seed=7), F)
    seen = []
    for _ in range(5):
        c.run()
        seen.append((c.loss.view.clone(), c.stats.view.clone(), c.grad.view.clone()))
    assert all(torch.equal(a, b) for s in seen[1:] for a, b in zip(s, seen[0]))


@pytest.mark.parametrize("prec,R,C", [(BF, 3300, 32769), (BF, 8300, 16384), (F, 13000, 4101), (F, 800, 70001), (BF, 30000, 4500)])
def test_more_than_the_caches_hold(gpu_lib, prec, R, C):
    # such calls go past the caches; the same rows, fewer at a time, do not: equal to the last bit
    K, es = 7, 2 if prec == BF else 4
    assert 2 * R * C * es > 400 << 20
    g = torch.Generator(device="cuda").manual_seed(R)
    z = Rows(R, C, dtype_of(prec), 0, 0, torch.randn(R, C, device="cuda", generator=g) * 3)
    ids = torch.randint(0, C, (R, K), device="cuda", generator=g, dtype=torch.int32)
    u = torch.randn(R, K, device="cuda", generator=g)
    weight = torch.rand(R, device="cuda", generator=g)

    def run(first, n):
        loss, stats = torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
        one, two = Rows(n, C, dtype_of(prec)), Rows(n, C, dtype_of(prec))
        head = (z.ptr + first * C * es, C, n, C, prec, ids[first:].data_ptr(), u[first:].data_ptr(), K, 2.0, weight[first:].data_ptr())
        fsb.fs_distill_device(*head, loss.data_ptr(), stats.data_ptr(), one.ptr, C, 0, stream())
        fsb.fs_distill_grad_device(*head, stats.data_ptr(), two.ptr, C, stream())
        assert one.untouched() and two.untouched()
        return loss, stats, one.view, two.view

    whole = run(0, R)
    for first in range(0, R, -(-R // 4)):
        n = min(R - first, -(-R // 4))
        for a, b in zip(whole, run(first, n)):
            assert torch.equal(a[first:first + n], b), first
    assert z.untouched()


def past_the_caches(R, C, K, prec, step):
    """Loss, statistics and both gradients of all rows and of a quarter at a time, equal to the last bit,
    and a few rows against the definition."""
    es = 2 if prec == BF else 4
    assert 2 * R * C * es > 400 << 20 >= 2 * -(-R // 4) * C * es
    g = torch.Generator(device="cuda").manual_seed(R + C)
    z = (torch.randn(R, C, device="cuda", generator=g) * 3).to(dtype_of(prec))
    ids = torch.randint(0, C, (R, K), device="cuda", generator=g, dtype=torch.int32)
    u = torch.randn(R, K, device="cuda", generator=g)
    weight = torch.rand(R, device="cuda", generator=g)

    def run(first, n):
        loss, stats = torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
        one, two = (torch.empty(n, C, dtype=z.dtype, device="cuda") for _ in range(2))
        head = (z[first:].data_ptr(), C, n, C, prec, ids[first:].data_ptr(), u[first:].data_ptr(), K, 2.0, weight[first:].data_ptr())
        fsb.fs_distill_device(*head, loss.data_ptr(), stats.data_ptr(), one.data_ptr() if step else 0, C, 0, stream())
        fsb.fs_distill_grad_device(*head, stats.data_ptr(), two.data_ptr(), C, stream())
        return (loss, stats, two) + ((one,) if step else ())

    whole = run(0, R)
    for first in range(0, R, -(-R // 4)):
        n = min(R - first, -(-R // 4))
        for a, b in zip(whole, run(first, n)):
            assert torch.equal(a[first:first + n], b), first
    for r in (0, R // 2, R - 1):
        c = Call(z[r:r + 1], ids[r:r + 1], u[r:r + 1], prec, 2.0)
        c.weight = weight[r:r + 1].contiguous()
        c.loss.view.copy_(whole[0][r])
        c.stats.view.copy_(whole[1][r])
        c.check_loss()
        for grad in whole[2:]:
            c.grad.view.copy_(grad[r])
            c.check_grad()


@pytest.mark.parametrize("prec,R,C,K", [(F, 40000, 1500, 128), (F, 52000, 1025, 5), (F, 26000, 2048, 128), (BF, 40000, 3001, 128), (BF, 26000, 4096, 64)])
def test_one_waves_gradient_past_the_caches(gpu_lib, prec, R, C, K):
    past_the_caches(R, C, K, prec, False)


# threads and the vectors of 16 bytes that each holds of a row, where the next larger kernel begins
HELD = [(64, 4), (128, 4), (128, 6), (256, 4), (256, 6), (256, 8), (256, 10), (256, 12), (256, 14), (256, 16), (512, 10), (512, 12),
        (512, 14), (512, 16), (512, 20), (512, 24), (512, 28), (512, 32)]


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("threads,held", HELD)
def test_rows_that_just_fit_a_workgroup(gpu_lib, threads, held, prec):
    most = threads * held * (8 if prec == BF else 4)
    for C in [most - 1, most - 3] + ([most] if held in (4, 16, 32) else []):
        Call(*inputs(3, C, 11), prec, 2.0, split=False).run().check_loss().check_grad()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("threads,held", HELD[4:])
def test_rows_that_just_fit_a_workgroup_past_the_caches(gpu_lib, threads, held, prec):
    C, es = threads * held * (8 if prec == BF else 4) - held // 2 % 2, 2 if prec == BF else 4
    past_the_caches((400 << 20) // (2 * C * es) + 9, C, 11, prec, True)
