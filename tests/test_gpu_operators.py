"""The operators together, as a program uses them next to an ensemble: the
ensemble's logits on the device give its alternatives; a small head's product
gives logits; the distillation loss and gradient fit the head to the ensemble."""
import numpy as np
import pytest
import torch

import workloads as wl
from oracle import operators as ref
from paper_2003_01538_amd import flexserve as fsb
from tests.device_rows import stream
from tests.test_gpu_logprob import near

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _teacher_logits(B):
    """[N][B][C] logits of the two tiny nets, on the device."""
    w = wl.workload("tiny2_fp32_b4")
    imgs = wl.images_uniform(w["image_seed"], B, *w["in_hw"])
    N, C = len(w["models"]), w["models"][0][-1]["cout"]
    with fsb.Ensemble(w["models"], w["out_hw"], wl.IMAGENET_MEAN, wl.IMAGENET_STD, "fp32", max_batch=B, device=0) as ens:
        pix = torch.from_numpy(np.stack(list(imgs))).cuda()
        h, wd = pix.shape[1:3]
        desc = np.zeros(B, np.dtype([("offset", "<u8"), ("h", "<i4"), ("w", "<i4"), ("stride", "<i4"), ("reserved", "<i4")]))
        desc["offset"], desc["h"], desc["w"], desc["stride"] = np.arange(B) * h * wd * 3, h, wd, 3 * wd
        d = torch.from_numpy(desc.view(np.uint8)).cuda()
        f = lambda *s: torch.empty(*s, device="cuda")
        probs, logits, top1 = f(N, B, C), f(N, B, C), torch.empty(N, B, dtype=torch.int32, device="cuda")
        vote = torch.empty(B, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        fsb.fs_infer_device(ens.handle, pix.data_ptr(), d.data_ptr(), B, probs.data_ptr(), 0, vote.data_ptr(), top1.data_ptr(),
                            logits.data_ptr(), stream())
        torch.cuda.synchronize()
    return logits, probs, top1


def test_an_ensembles_alternatives_train_a_head(gpu_lib):
    B, K, feat = 4, 3, 24
    logits, probs, top1 = _teacher_logits(B)
    N, _, C = logits.shape
    R = N * B
    f = lambda *s: torch.empty(*s, device="cuda")
    # the ensemble's answers as alternatives
    ids, best, ent = torch.empty(R, K, dtype=torch.int32, device="cuda"), f(R, K), f(R)
    logp = f(R, 1)
    given = top1.reshape(R, 1).contiguous()
    scratch = torch.empty(fsb.FS_ROW_SCRATCH_BYTES, dtype=torch.uint8, device="cuda")
    fsb.fs_logprob_device(logits.data_ptr(), C, R, C, fsb.FS_F32, given.data_ptr(), 1, K, logp.data_ptr(), ent.data_ptr(),
                          ids.data_ptr(), best.data_ptr(), scratch.data_ptr(), stream())
    assert torch.equal(ids[:, :1], given) and torch.equal(best[:, :1], logp)
    p = probs.reshape(R, C).cpu().numpy().astype(np.float64)
    near(np.exp(best.cpu().numpy().astype(np.float64)), np.take_along_axis(p, ids.cpu().numpy().astype(np.int64), 1), lambda v: 2e-6)
    # a head of its own on shared features, trained towards them with plain descent
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(R, feat, device="cuda", generator=g)
    w, b = torch.randn(C, feat, device="cuda", generator=g) * 0.2, torch.zeros(C, device="cuda")
    for step in range(3):
        z, loss, grad = f(R, C), f(R), f(R, C)
        fsb.fs_linear_device(x.data_ptr(), feat, w.data_ptr(), feat, b.data_ptr(), 0, 0, z.data_ptr(), C, R, C, feat, fsb.FS_F32,
                             fsb.FS_F32, fsb.FS_ACT_NONE, 0, stream())
        weight = torch.full((R,), 1.0 / R, device="cuda")
        fsb.fs_distill_device(z.data_ptr(), C, R, C, fsb.FS_F32, ids.data_ptr(), best.data_ptr(), K, 2.0, weight.data_ptr(),
                              loss.data_ptr(), 0, grad.data_ptr(), C, scratch.data_ptr(), stream())
        # against the chain in 64 bits from the same weights
        zw, size = ref.linear(x.cpu().numpy(), w.cpu().numpy(), b.cpu().numpy())
        assert (np.abs(z.cpu().numpy() - zw) <= (2 * feat + 24) * U * size).all()
        want = ref.distill(z.cpu().numpy(), ids.cpu().numpy(), best.cpu().numpy(), 2.0, weight.cpu().numpy())
        near(loss.cpu().numpy(), want["loss"], lambda v: (256 + 8 * 20) * U + 8 * U * np.abs(v))
        near(grad.cpu().numpy(), want["grad"], lambda v: 128 * U / R)
        w -= 1.0 * grad.t() @ x
        b -= 1.0 * grad.sum(0)
