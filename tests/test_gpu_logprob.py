"""fs_logprob_device against the definition in 64 bits.

Tolerances, in steps of U = 2^-24: the sum of exponentials is off by some 32 steps
of itself (each term by a few, the tree by one per level and the runs of a thread
by one per term, of independent signs), its logarithm by as many absolute steps and
two of itself; z - m and the difference of the two by one step of themselves.
So ln p is within (128 + 8 |ln p|) U, and the entropy, whose second part is a
quotient of two such sums of at most ln C, within (128 + 48 (1 + ln C)) U.
Classes of the alternatives are exact."""
import math

import numpy as np
import pytest
import torch

from oracle import operators as ref
from paper_2003_01538_amd import flexserve as fsb
from tests.device_rows import Rows, dtype_of, stream

pytestmark = pytest.mark.gpu
BF, F = fsb.FS_BF16, fsb.FS_F32
U = 2.0 ** -24


def scratch():
    return torch.empty(fsb.FS_ROW_SCRATCH_BYTES, dtype=torch.uint8, device="cuda")


class Call:
    def __init__(self, z, prec, T, K, classes=None, pad=0, lead=0, split=True, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        R, C = z.shape
        self.z, self.prec, self.T, self.K = Rows(R, C, dtype_of(prec), pad, lead, z), prec, T, K
        self.classes = torch.randint(0, C, (R, T), device="cuda", generator=g, dtype=torch.int32) if classes is None else \
            classes.to(device="cuda", dtype=torch.int32)
        self.logp, self.entropy = Rows(R, T, torch.float32), Rows(R, 1, torch.float32)
        self.ids, self.best = Rows(R, K, torch.int32), Rows(R, K, torch.float32)
        self.scratch = scratch() if split else None

    def run(self, st=None):
        z = self.z
        fsb.fs_logprob_device(z.ptr, z.ld, z.rows, z.cols, self.prec, self.classes.data_ptr() if self.T else 0, self.T, self.K,
                              self.logp.ptr if self.T else 0, self.entropy.ptr, self.ids.ptr if self.K else 0,
                              self.best.ptr if self.K else 0, self.scratch.data_ptr() if self.scratch is not None else 0,
                              stream() if st is None else st)
        return self

    def check(self):
        z = self.z
        want = ref.logprob(z.numpy(), self.classes.cpu().numpy(), self.K)
        assert np.array_equal(self.ids.numpy(), want["top_ids"])
        near(self.logp.numpy(), want["logp"], lambda v: (128 + 8 * np.abs(v)) * U)
        near(self.best.numpy(), want["top_logp"], lambda v: (128 + 8 * np.abs(v)) * U)
        near(self.entropy.numpy()[:, 0], want["entropy"], lambda v: (128 + 48 * (1 + math.log(z.cols))) * U)
        assert all(t.untouched() for t in (z, self.logp, self.entropy, self.ids, self.best))
        return self


def near(got, want, tol):
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        ok = np.isfinite(want) & np.isfinite(got) & (np.abs(got.astype(np.float64) - want) <= tol(want))
    assert (same | ok).all(), (got[~(same | ok)][:4], want[~(same | ok)][:4])


def logits(R, C, seed, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + R + C)
    return torch.randn(R, C, device="cuda", generator=g) * spread


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("R,C,T,K", [
    (1, 1, 1, 1), (1, 2, 3, 5), (3, 10, 1, 5), (2, 63, 2, 63), (5, 64, 1, 64), (4, 65, 1, 128), (96, 1000, 1, 5),
    (7, 1001, 2, 20), (2, 4096, 1, 20), (1, 4097, 4, 128), (3, 8191, 1, 1), (1, 20000, 1, 20), (33, 16385, 1, 10),
    (1, 131072, 1, 64), (2, 100003, 300, 128), (700, 257, 1, 3), (1, 262144, 0, 20), (5, 30000, 2, 0), (300, 9000, 1, 7),
])
def test_sizes(gpu_lib, R, C, T, K, prec, split):
    Call(logits(R, C, 1), prec, T, K, split=split).run().check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("pad,lead", [(0, 1), (1, 0), (3, 2), (4, 4), (8, 8), (2, 6), (7, 5)])
@pytest.mark.parametrize("R,C", [(3, 50), (2, 5001), (1, 70000), (70, 1003)])
def test_strides_and_alignment(gpu_lib, R, C, pad, lead, prec):
    c = Call(logits(R, C, 2), prec, 1, 9, pad=pad, lead=lead)
    keep = c.z.view.clone()
    c.z.buf.fill_(1e30)  # beside the rows: read into no row
    c.z.view.copy_(keep)
    c.run()
    c.z.buf.fill_(7.25)
    c.z.view.copy_(keep)
    c.check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("C", [7, 1000, 5000, 40000, 150000])
def test_masks_and_values_that_are_not_finite(gpu_lib, C, prec):
    inf, nan = float("inf"), float("nan")
    low = torch.finfo(dtype_of(prec)).min
    z = logits(14, C, 3)
    g = torch.Generator(device="cuda").manual_seed(C)
    z[0] = -inf                                                # nothing left
    z[1] = -inf
    z[1, C - 1] = 2.0                                          # one class left
    z[2, torch.rand(C, device="cuda", generator=g) < 0.9] = -inf
    z[3] = low                                                 # the lowest value everywhere: a uniform row
    z[4, torch.rand(C, device="cuda", generator=g) < 0.9] = low
    z[5] = -inf
    z[5, C // 2] = low                                         # the lowest value alone
    z[6, C // 3] = nan
    z[7, C // 3] = inf
    z[8] = nan
    z[9, 0] = -nan
    z[9, 1] = -inf
    z[10] = -1e4
    z[10, 3] = 1e4
    z[11] = 0.0
    z[11, ::2] = -0.0                                          # equal to 0: ties by class
    z[12, : C // 2] = -inf                                     # whole chunks masked, the first ones
    z[13] = -torch.arange(C, device="cuda") / C * 50
    cls = torch.tensor([[0, C - 1, -1, C]] * 14)
    for split in (True, False):
        Call(z, prec, 4, 6, classes=cls, split=split).run().check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("C", [300, 5000, 33000, 140000])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "few", "steps", "late"])
def test_orders_that_are_hard_for_a_selection(gpu_lib, C, kind, prec):
    i = torch.arange(C, device="cuda", dtype=torch.float32)
    z = {"rising": i / C * 40 - 20, "falling": -i / C * 40, "equal": torch.full((C,), 1.5, device="cuda"),
         "few": torch.where(i % 1000 == 7, 3.0, 0.0), "steps": torch.floor(i / 700), "late": torch.where(i > C - 200, 5.0, 0.0)}[kind]
    z = torch.stack([z, z.flip(0), z.roll(C // 3)])
    for K in (1, 37, 128):
        Call(z, prec, 1, K).run().check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("C", [900, 5000, 33000, 140000])
def test_many_infinities(gpu_lib, C, prec):
    # more candidates than a list holds, all of them at the largest logit there is
    inf = float("inf")
    z = logits(4, C, 10)
    z[0] = inf
    z[1, ::2] = inf
    z[2, C // 2:] = inf
    z[3, ::3] = torch.finfo(torch.float32).max if prec == F else torch.finfo(torch.bfloat16).max
    for K in (1, 50, 128):
        Call(z, prec, 1, K).run().check()


def test_wave_rows_with_many_alternatives(gpu_lib):
    for K in (39, 40, 41, 64, 65, 128):
        Call(logits(30, 1000, 11), F, 1, K).run().check()


@pytest.mark.parametrize("R", [255, 256, 511, 512, 1023, 1024])
def test_row_counts_around_the_rules(gpu_lib, R):
    Call(logits(R, 5000, 12), F, 1, 3).run().check()
    Call(logits(R, 16400, 12), BF, 1, 3).run().check()


def test_large_logits_keep_their_differences(gpu_lib):
    z = logits(4, 3000, 4)
    for shift in (1000.0, -30000.0):
        Call(z + shift, F, 1, 5).run().check()


def test_ensemble_rows_at_a_32_bit_offset(gpu_lib):
    # the rows of a buffer of more than 2^32 bytes: the last rows start behind 2^31 elements
    C, R = 1 << 20, 2100
    big = torch.zeros(R * C, device="cuda").view(R, C)
    last = logits(2, C, 5)
    big[R - 2:] = last
    f = lambda *s: torch.empty(*s, device="cuda")
    ids, best, ent = torch.empty(R, 3, dtype=torch.int32, device="cuda"), f(R, 3), f(R)
    fsb.fs_logprob_device(big.data_ptr(), C, R, C, F, 0, 0, 3, 0, ent.data_ptr(), ids.data_ptr(), best.data_ptr(), 0, stream())
    want = ref.logprob(last.cpu().numpy(), np.zeros((2, 0), int), 3)
    assert np.array_equal(ids[R - 2:].cpu().numpy(), want["top_ids"])
    near(best[R - 2:].cpu().numpy(), want["top_logp"], lambda v: (128 + 8 * np.abs(v)) * U)
    assert (ids[: R - 2] == torch.arange(3, device="cuda")).all() and torch.allclose(ent[: R - 2], torch.tensor(math.log(C)).cuda())


@pytest.mark.parametrize("R,C", [(3, 900), (2, 5000), (3, 70000)])
def test_outputs_that_are_not_asked_for(gpu_lib, R, C):
    full = Call(logits(R, C, 14), F, 2, 7).run()
    z, sc = full.z, full.scratch.data_ptr()
    logp, ent, best, ids = (torch.full_like(t.view, t.mark()) for t in (full.logp, full.entropy, full.best, full.ids))
    head = (z.ptr, z.ld, R, C, F)
    fsb.fs_logprob_device(*head, full.classes.data_ptr(), 2, 0, logp.data_ptr(), 0, 0, 0, sc, stream())
    fsb.fs_logprob_device(*head, 0, 0, 7, 0, 0, ids.data_ptr(), best.data_ptr(), sc, stream())
    fsb.fs_logprob_device(*head, 0, 0, 0, 0, ent.data_ptr(), 0, 0, sc, stream())
    for got, want in ((logp, full.logp), (ent, full.entropy), (best, full.best), (ids, full.ids)):
        assert torch.equal(got, want.view)


def test_more_rows_than_workgroups(gpu_lib):
    R, C, K = (1 << 20) + 70, 5, 3
    z = logits(R, C, 13)
    f = lambda *s: torch.empty(*s, device="cuda")
    cls = (torch.arange(R, device="cuda") % C).int()
    logp, ent, best, ids = f(R), f(R), f(R, K), torch.empty(R, K, dtype=torch.int32, device="cuda")
    fsb.fs_logprob_device(z.data_ptr(), C, R, C, F, cls.data_ptr(), 1, K, logp.data_ptr(), ent.data_ptr(), ids.data_ptr(), best.data_ptr(),
                          0, stream())
    lp = torch.log_softmax(z.double(), 1)
    v, i = torch.sort(z, dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), i[:, :K])
    for got, want in ((logp, lp.gather(1, cls.long()[:, None])[:, 0]), (best, lp.gather(1, i[:, :K]))):
        assert bool(((got.double() - want).abs() <= (128 + 8 * want.abs()) * U).all())
    assert bool(((ent.double() + (lp.exp() * lp).sum(1)).abs() <= (128 + 48 * (1 + math.log(C))) * U).all())


def test_two_streams_with_scratch_of_their_own(gpu_lib):
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    one, two = Call(logits(1, 131072, 6), F, 1, 20), Call(logits(3, 90000, 7), BF, 1, 50)
    torch.cuda.synchronize()
    for _ in range(10):
        one.run(a.cuda_stream)
        two.run(b.cuda_stream)
    torch.cuda.synchronize()
    one.check()
    two.check()


@pytest.mark.parametrize("R,C", [(2, 130000), (96, 1000)])
def test_captured_and_replayed(gpu_lib, R, C):
    # two graphs share one scratch and run in turn on one stream
    s = torch.cuda.Stream()
    calls = [Call(logits(R, C, 8 + i), F, 1, 12) for i in range(2)]
    calls[1].scratch = calls[0].scratch
    graphs = []
    for c in calls:
        c.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            c.run(s.cuda_stream)
        graphs.append(g)
    for i in range(4):
        for c in calls:
            c.z.view.copy_(c.z.view.roll(37, 1))
            for t in (c.logp, c.entropy, c.ids, c.best):
                t.view.fill_(t.mark())
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for c in calls:
            c.check()


def test_same_bits_every_time(gpu_lib):
    c = Call(logits(3, 131072, 9), F, 1, 64)
    seen = []
    for _ in range(5):
        c.run()
        seen.append((c.entropy.view.clone(), c.best.view.clone(), c.ids.view.clone()))
    assert all(torch.equal(a, b) for s in seen[1:] for a, b in zip(s, seen[0]))


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("R,C", [(99, 17000), (100, 17000), (199, 33000), (200, 33000)])
def test_row_counts_around_the_split(gpu_lib, R, C, prec):
    Call(logits(R, C, 13), prec, 2, 20).run().check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("C", [1, 37, 100, 255, 256, 257, 511, 512, 513, 600])
def test_short_rows(gpu_lib, C, prec):
    for K in (1, 20, 48, 49, 80, 81, 128):
        Call(logits(33, C, 14), prec, 1, K, pad=C % 3).run().check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("R,C,K", [(1999, 2100, 5), (2000, 2100, 5), (2000, 2100, 80), (2000, 2100, 81), (3999, 2100, 48), (4000, 2100, 48), (4000, 2100, 49)])
def test_many_rows(gpu_lib, R, C, K, prec):
    Call(logits(R, C, 15), prec, 1, K).run().check()


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("K", [1, 37, 70])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "few", "steps", "late"])
def test_orders_that_are_hard_for_a_wave(gpu_lib, kind, K, prec):
    # more rows than are given four waves; all alike, so that one is compared and the others with it
    C, R = 9000, 4000
    i = torch.arange(C, device="cuda", dtype=torch.float32)
    z = {"rising": i / C * 40 - 20, "falling": -i / C * 40, "equal": torch.full((C,), 1.5, device="cuda"),
         "few": torch.where(i % 1000 == 7, 3.0, 0.0), "steps": torch.floor(i / 700), "late": torch.where(i > C - 200, 5.0, 0.0)}[kind]
    one = Call(z[None], prec, 1, K, classes=torch.tensor([[5]])).run().check()
    all_ = Call(z[None].expand(R, C), prec, 1, K, classes=torch.full((R, 1), 5)).run()
    assert bool((all_.ids.view == one.ids.view).all())
    # another split of the same sums: the two are each within the tolerance of check()
    near(all_.best.numpy(), np.broadcast_to(one.best.numpy(), (R, K)), lambda v: 2 * (256 + 8 * 20) * U + 16 * U * np.abs(v))


@pytest.mark.parametrize("prec,R,C,K", [(F, 4100, 26000, 9), (BF, 2100, 101000, 20), (F, 1100, 100001, 30), (F, 4400, 24001, 100)])
def test_more_than_the_caches_hold(gpu_lib, prec, R, C, K):
    # such calls go past the caches; a few of their rows against the definition, the others' alternatives by sorting
    z = logits(R, C, 16)
    assert R * C * (2 if prec == BF else 4) > 400 << 20
    c = Call(z, prec, 1, K).run()
    for r in (0, R // 2, R - 1):
        want = ref.logprob(c.z.numpy()[r:r + 1], c.classes[r:r + 1].cpu().numpy(), K)
        assert np.array_equal(c.ids.numpy()[r:r + 1], want["top_ids"])
        near(c.logp.numpy()[r:r + 1], want["logp"], lambda v: (128 + 8 * np.abs(v)) * U)
        near(c.entropy.numpy()[r:r + 1, 0], want["entropy"], lambda v: (128 + 48 * (1 + math.log(C))) * U)
    top = c.z.view.float().sort(dim=1, descending=True, stable=True)
    assert torch.equal(c.ids.view, top.indices[:, :K].int())


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("K", [1, 48, 49, 80])
@pytest.mark.parametrize("kind", ["rising", "falling", "equal", "few", "steps", "late"])
def test_hard_orders_by_one_and_two_waves_against_the_definition(gpu_lib, kind, K, prec):
    # rows of one and of two waves (K beyond 48), the orders shifted from row to row
    C, R = 9000, 4000
    i = torch.arange(C, device="cuda", dtype=torch.float32)
    z = {"rising": i / C * 40 - 20, "falling": -i / C * 40, "equal": torch.full((C,), 1.5, device="cuda"),
         "few": torch.where(i % 1000 == 7, 3.0, 0.0), "steps": torch.floor(i / 700), "late": torch.where(i > C - 200, 5.0, 0.0)}[kind]
    z = z[(torch.arange(C, device="cuda")[None] + 37 * torch.arange(R, device="cuda")[:, None]) % C]
    c = Call(z, prec, 1, K).run()
    at = [0, 1, 243, 1999, R - 1]
    want = ref.logprob(c.z.view[at].float().cpu().numpy(), c.classes[at].cpu().numpy(), K)
    assert np.array_equal(c.ids.numpy()[at], want["top_ids"])
    near(c.logp.numpy()[at], want["logp"], lambda v: (128 + 8 * np.abs(v)) * U)
    near(c.best.numpy()[at], want["top_logp"], lambda v: (128 + 8 * np.abs(v)) * U)
    near(c.entropy.numpy()[at, 0], want["entropy"], lambda v: (128 + 48 * (1 + math.log(C))) * U)
    assert torch.equal(c.ids.view, c.z.view.float().sort(dim=1, descending=True, stable=True).indices[:, :K].int())


@pytest.mark.parametrize("prec", [BF, F])
@pytest.mark.parametrize("C", [37, 100, 255, 256, 257, 511, 512, 513])
@pytest.mark.parametrize("K", [49, 81, 128])
def test_many_short_rows_with_many_alternatives(gpu_lib, C, K, prec):
    z = logits(4100, C, 17)
    z[:50] = torch.floor(z[:50])  # ties
    z[50:60, C // 3:] = -float("inf")
    z[60:64] = 1.0
    c = Call(z, prec, 2, K, pad=C % 3).run()
    at = [0, 7, 49, 50, 59, 60, 64, 2000, 4099]
    want = ref.logprob(c.z.view[at].float().cpu().numpy(), c.classes[at].cpu().numpy(), K)
    assert np.array_equal(c.ids.numpy()[at], want["top_ids"])
    near(c.logp.numpy()[at], want["logp"], lambda v: (128 + 8 * np.abs(v)) * U)
    near(c.best.numpy()[at], want["top_logp"], lambda v: (128 + 8 * np.abs(v)) * U)
    near(c.entropy.numpy()[at, 0], want["entropy"], lambda v: (128 + 48 * (1 + math.log(C))) * U)
    v, i = c.z.view.float().sort(dim=1, descending=True, stable=True)
    n = min(K, C)
    assert torch.equal(c.ids.view[:, :n], torch.where(v == -float("inf"), -1, i)[:, :n].int())
    assert bool((c.ids.view[:, n:] == -1).all()) and all(t.untouched() for t in (c.logp, c.entropy, c.ids, c.best))
