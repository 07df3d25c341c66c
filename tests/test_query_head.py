"""The head of learned queries on the CPU: sizes, outputs and refusals through the C ABI."""
import numpy as np
import pytest
import torch

import paper_2508_11584_amd as vpe
import vpe_inputs as vi
from helpers import make_engine

SPEC = vi.with_(vi.small_spec(), batch=2, det_classes=7, head_ch=64)


def host_engine(spec=SPEC, kinds=("query",)):
    return make_engine(spec, 1, kinds=kinds, flags=vpe.VPE_FLAG_HOST_ONLY)[0]


def test_runs_are_counted_and_the_output_is_a_row_of_logits_a_query():
    eng = host_engine(kinds=("seg", "query"))
    fh = eng.encode(None)
    assert eng.run_head(1, fh) == vpe.VPE_OK and eng.run_head_static(1, fh) == vpe.VPE_OK
    assert eng.stats()[1] == [0, 2]
    assert vpe.vpe_head_output(eng.handle, 1, 0)[1] == (2, 64, 7, 1)
    with pytest.raises(vpe.VpeError, match="no such output"):
        vpe.vpe_head_output(eng.handle, 1, 1)


@pytest.mark.parametrize("channels,classes,ok", [(1, 1, True), (3, 256, True), (256, 2, True), (0, 2, False), (257, 2, False), (4, 0, False), (4, 257, False)])
def test_sizes(channels, classes, ok):
    spec = vi.with_(SPEC, head_ch=channels, det_classes=classes)
    if ok:
        eng = host_engine(spec)
        assert vpe.vpe_head_output(eng.handle, 0, 0)[1] == (2, channels, classes, 1)
    else:
        with pytest.raises(vpe.VpeError, match="queries" if classes == 2 else "classes"):
            host_engine(spec)


def test_a_blob_of_another_size_is_refused():
    hw = vi.make_head_weights(SPEC, vi.HEAD_QUERY, 1)
    blob = vi.pack_head(SPEC, vi.HEAD_QUERY, hw)
    D = SPEC.dim
    assert blob.size == 64 * D + 4 * D * D + 4 * D + 3 * D + 7 * D + 7
    with pytest.raises(vpe.VpeError, match="weights_bytes"):
        w = vi.make_backbone_weights(SPEC, 1)
        vpe.Engine(dim=D, depth=SPEC.depth, heads=SPEC.heads, mlp_hidden=SPEC.mlp_hidden, img_h=SPEC.img_h, img_w=SPEC.img_w, batch=2, taps=SPEC.taps,
                   mlp_kind=SPEC.mlp_kind, registers=SPEC.registers, weights=vi.pack_backbone(SPEC, w), flags=vpe.VPE_FLAG_HOST_ONLY,
                   head_cfgs=[vpe.HeadCfg(kind=vpe.VPE_HEAD_QUERY, weights=blob[:-1], classes=7, channels=64)])


def test_adapters_are_checked():
    eng = host_engine(kinds=("seg", "query"))
    D = SPEC.dim
    dtype = torch.bfloat16 if SPEC.dtype == "bf16" else torch.float32
    a, b = torch.zeros(2, 16, D, dtype=dtype), torch.zeros(2, 2 * D, 16, dtype=dtype)
    eng.set_head_adapters(1, a, b, (0, -1), scale=torch.ones(2))
    eng.set_head_adapters(1)
    with pytest.raises(vpe.VpeError, match="takes no adapters"):
        eng.set_head_adapters(0, a, b, (0, 1))
    with pytest.raises(vpe.VpeError, match="unknown head"):
        eng.set_head_adapters(2, a, b, (0, 1))
    with pytest.raises(vpe.VpeError, match="image"):
        eng.set_head_adapters(1, a, b, (0,))
    with pytest.raises(vpe.VpeError, match="null"):
        eng.set_head_adapters(1, a, None, (0, 1))
    with pytest.raises(vpe.VpeError, match="b: contiguous"):
        eng.set_head_adapters(1, a, b[:, :D], (0, 1))
    with pytest.raises(vpe.VpeError, match="scale"):
        eng.set_head_adapters(1, a, b, (0, 1), scale=torch.ones(3))
    eng.set_head_adapters(1, a, b, (2 ** 40, -2 ** 40))          # (no index of an adapter: the images have none)
    call = dict(engine=eng.handle, head=1, adapters=2, rank=16, a_ptr=4096, b_ptr=8192, scale_ptr=None, adapter_of_image=(0, 1))
    vpe.vpe_set_head_adapters(**call)
    for over, needle in [(dict(rank=12), "rank"), (dict(rank=0), "rank"), (dict(rank=136), "rank"), (dict(adapters=-1), "negative"), (dict(a_ptr=None), "null"),
                         (dict(a_ptr=4104), "aligned"), (dict(b_ptr=4098), "aligned"), (dict(scale_ptr=4097), "aligned")]:
        with pytest.raises(vpe.VpeError, match=needle):
            vpe.vpe_set_head_adapters(**{**call, **over})


def test_weights_are_named_and_drawn_like_those_of_other_heads():
    hw = vi.make_head_weights(SPEC, vi.HEAD_QUERY, 3)
    assert np.allclose(hw["ls1"], 0.1, atol=1e-3) and abs(float(hw["norm_g"].mean()) - 1) < 0.05
    assert hw["kv_w"].shape == (2 * SPEC.dim, SPEC.dim) and hw["query"].shape == (64, SPEC.dim)
