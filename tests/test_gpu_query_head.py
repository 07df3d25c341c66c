"""The head of learned queries on the GPU, against the same computation in 64 bits from the features that it read."""
import pytest
import torch

import paper_2508_11584_amd as vpe
import vpe_inputs as vi
from helpers import make_engine

pytestmark = pytest.mark.gpu

BASE = vi.ModelSpec("query", dim=128, depth=4, heads=2, mlp_hidden=256, img_h=98, img_w=154, taps=(1, 2, 3, 4), head_ch=64, det_classes=11, dtype="bf16", batch=2)


def expected(spec, w, feat, adapters=None):
    """(logits, bound of their error), both 64-bit [B, Q, C].  The bound carries every rounding to the engine's type (half a step, U) and the
    32-bit sums (2^-24 a term and for each of the terms' own roundings) through the head's steps to first order; products of errors are
    covered by the 2 in front at the end."""
    f64 = torch.float64
    w = {k: torch.from_numpy(v.copy()).to(f64) for k, v in w.items() if k != "__blob__"}
    B, Q, D, H = spec.batch, spec.head_ch, spec.dim, spec.heads
    U = torch.finfo(torch.bfloat16 if spec.dtype == "bf16" else torch.float32).eps / 2

    def sums(terms):
        return (terms + 16) * 2.0 ** -24

    def linear(x, ex, weight, bias, rounded=True):
        y = x @ weight.T + bias
        size = x.abs() @ weight.abs().T + bias.abs()
        e = ex @ weight.abs().T + sums(x.shape[-1]) * size
        return y, e + (U * y.abs() if rounded else 0)

    m = feat.to("cpu", f64)                                            # [B, N, D]
    kv, ekv = linear(m, torch.zeros_like(m), w["kv_w"], w["kv_b"])
    if adapters is not None:
        a, b, scale, of = adapters
        for i, k in enumerate(of):
            if 0 <= k < a.shape[0]:
                ak, bk, s = a[k].to("cpu", f64), b[k].to("cpu", f64), 1.0 if scale is None else float(scale[k])
                low = m[i] @ ak.T
                elow = (2.0 ** -16 + sums(D)) * (m[i].abs() @ ak.abs().T)          # carried in 16 bits or more
                more = s * (low @ bk.T)
                kv[i] += more
                ekv[i] += abs(s) * (elow @ bk.abs().T + sums(ak.shape[0]) * (low.abs() @ bk.abs().T)) + U * more.abs()
    t = w["query"]
    q = t @ w["q_w"].T + w["q_b"]
    eq = U * q.abs() + 2.0 ** -24 * q.abs()

    def heads(x):
        return x.reshape(x.shape[0], -1, H, 64).permute(0, 2, 1, 3) if x.dim() == 3 else x.reshape(-1, H, 64).permute(1, 0, 2)

    k, v, ek, ev = heads(kv[..., :D]), heads(kv[..., D:]), heads(ekv[..., :D]), heads(ekv[..., D:])
    q, eq = heads(q)[None].expand(B, -1, -1, -1), heads(eq)[None].expand(B, -1, -1, -1)
    s = q @ k.transpose(-1, -2) / 8
    size = q.abs() @ k.abs().transpose(-1, -2) / 8
    es = (q.abs() @ ek.transpose(-1, -2) + eq @ k.abs().transpose(-1, -2)) / 8 + sums(64) * size + 2.0 ** -22 * s.abs()
    p = torch.softmax(s, -1)
    r = torch.expm1(2 * es.amax(-1, keepdim=True)) + U + 2.0 ** -20 + sums(k.shape[-2])     # (a weight, and their sum)
    att = p @ v
    eatt = r * (p @ v.abs()) + p @ ev + U * att.abs()
    att, eatt = (x.permute(0, 2, 1, 3).reshape(B, Q, D) for x in (att, eatt))
    y, ey = linear(att, eatt, w["out_w"], w["out_b"])
    x = t + w["ls1"] * y
    ex = w["ls1"].abs() * ey + 2.0 ** -22 * (t.abs() + x.abs())
    mu = x.mean(-1, keepdim=True)
    sigma = ((x - mu).pow(2).mean(-1, keepdim=True) + spec.ln_eps).sqrt()
    xh = (x - mu) / sigma
    n = xh * w["norm_g"] + w["norm_b"]
    en = w["norm_g"].abs() * ((ex + ex.mean(-1, keepdim=True) + xh.abs() * (xh.abs() * ex).mean(-1, keepdim=True)) / sigma
                              + sums(D) * (xh.abs() + (mu / sigma).abs() + 1)) + (U + 2.0 ** -22) * n.abs()
    out, e = linear(n, en, w["cls_w"], w["cls_b"], rounded=False)
    return out, 2 * e + 1e-30


def check(eng, head, spec, w, fh, adapters=None):
    got = eng.head_output(head, 0).double().cpu()
    ref, bound = expected(spec, w, eng.feat_view(fh, 3), adapters)
    assert got.shape == ref.shape
    off = (got - ref).abs() / bound
    assert torch.isfinite(got).all() and off.max() <= 1, f"largest error is {off.max():.2f} of its bound"


def draw_adapters(spec, n, rank, seed):
    g = torch.Generator().manual_seed(seed)
    dtype = torch.bfloat16 if spec.dtype == "bf16" else torch.float32
    a = (torch.randn(n, rank, spec.dim, generator=g) * 0.2).to(dtype).cuda()
    b = (torch.randn(n, 2 * spec.dim, rank, generator=g) * 0.2).to(dtype).cuda()
    return a, b, torch.linspace(-0.5, 1.0, n).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("queries,classes,batch,registers", [(1, 1, 1, 0), (5, 11, 2, 3), (64, 256, 1, 0), (256, 3, 3, 1)])
def test_logits(dtype, queries, classes, batch, registers):
    spec = vi.with_(BASE, dtype=dtype, head_ch=queries, det_classes=classes, batch=batch, registers=registers)
    eng, _, hd = make_engine(spec, 31, kinds=("query",))
    fh = eng.encode(torch.from_numpy(vi.make_batch(spec, 32)).cuda())
    assert eng.run_head(0, fh) == vpe.VPE_OK
    eng.sync()
    check(eng, 0, spec, hd[0], fh)


@pytest.mark.parametrize("img,heads", [((14, 14), 2), ((14, 28), 1), ((420, 560), 6)])
def test_logits_of_small_and_large_images(img, heads):
    spec = vi.with_(BASE, img_h=img[0], img_w=img[1], dim=64 * heads, heads=heads, batch=1, head_ch=17)
    eng, _, hd = make_engine(spec, 41, kinds=("query",))
    fh = eng.encode(torch.from_numpy(vi.make_batch(spec, 42)).cuda())
    assert eng.run_head(0, fh) == vpe.VPE_OK
    eng.sync()
    check(eng, 0, spec, hd[0], fh)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("flags", [0, vpe.VPE_FLAG_GRAPHS])
def test_adapters_of_images_change_between_runs(dtype, flags):
    spec = vi.with_(BASE, dtype=dtype, batch=3, head_ch=9)
    eng, _, hd = make_engine(spec, 51, kinds=("seg", "query"), flags=flags)
    a, b, scale = draw_adapters(spec, 2, 24, 52)
    choices = [None, (a, b, scale, (1, -1, 0)), (a, b, None, (0, 0, 5)), (a[:1].contiguous(), b[:1].contiguous(), scale[:1].contiguous(), (0, -7, 0)), None]
    for step, adapters in enumerate(choices):
        if adapters is None:
            eng.set_head_adapters(1)
        else:
            eng.set_head_adapters(1, adapters[0], adapters[1], adapters[3], scale=adapters[2])
        for again in range(3):                 # both ring slots, and one of them replayed
            fh = eng.encode(torch.from_numpy(vi.make_batch(spec, 60 + 3 * step + again)).cuda())
            assert eng.run_head(0, fh) == vpe.VPE_OK and eng.run_head(1, fh) == vpe.VPE_OK
            eng.sync()
            check(eng, 1, spec, hd[1], fh, adapters)


def test_the_static_run_and_a_stream_of_the_callers_give_the_same_bits():
    spec = vi.with_(BASE, head_ch=33)
    eng, _, hd = make_engine(spec, 71, kinds=("query",))
    a, b, scale = draw_adapters(spec, 3, 128, 72)
    eng.set_head_adapters(0, a, b, (2, 0), scale=scale)
    fh = eng.encode(torch.from_numpy(vi.make_batch(spec, 73)).cuda())
    assert eng.run_head(0, fh) == vpe.VPE_OK
    eng.sync()
    ref = eng.head_output(0, 0).clone()
    check(eng, 0, spec, hd[0], fh, (a, b, scale, (2, 0)))
    stream = torch.cuda.Stream()
    for run in (lambda: eng.run_head_static(0, fh), lambda: eng.run_head(0, fh, stream)):
        eng.head_output(0, 0).fill_(7)
        torch.cuda.synchronize()
        assert run() == vpe.VPE_OK
        eng.sync()
        assert torch.equal(eng.head_output(0, 0), ref)
