"""What the operators on packed rows refuse, and the workspaces they ask for: decided from the arguments alone, with a device or without."""
import ctypes as C

import pytest

import paper_2508_11584_amd as vpe
from paper_2508_11584_amd import binding

PTR = 1 << 20                                    # an aligned address; a refused call never uses it


def attention_args(**kw):
    a = vpe.vpe_attention_args()
    base = dict(dtype=vpe.VPE_BF16, heads=8, kv_heads=2, head_dim=64, sequences=2, max_q=10, max_k=20, q_rows=15, k_rows=40, causal=0, scale=0.125,
                cap=0.0, q=PTR, k=PTR, v=PTR, out=PTR, q_row=512, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, out_row=512, out_head=64,
                q_offsets=PTR, k_offsets=PTR)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def norm_args(**kw):
    a = vpe.vpe_block_norm_args()
    base = dict(dtype=vpe.VPE_BF16, rows=5, dim=100, requests=2, post=1, pre=2, residual_scale=1.0, eps=1e-6, x=PTR, branch=PTR, out=PTR + (1 << 16), normed=PTR,
                x_row=100, branch_row=100, out_row=100, normed_row=100)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def adapter_args(**kw):
    a = vpe.vpe_adapter_linear_args()
    base = dict(dtype=vpe.VPE_BF16, out_f32=0, rows=5, in_features=128, out_features=100, adapters=3, rank=16, x=PTR, weight=PTR, out=PTR, x_row=128,
                out_row=100, a=PTR, b=PTR, adapter=PTR, workspace=PTR, workspace_bytes=1 << 30)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


NAN, INF = float("nan"), float("inf")
REFUSED = [
    ("vpe_attention", attention_args, kw) for kw in (
        dict(dtype=2), dict(dtype=-1), dict(head_dim=32), dict(head_dim=0), dict(head_dim=96), dict(heads=0), dict(heads=7), dict(kv_heads=0), dict(kv_heads=-2),
        dict(heads=8192, kv_heads=1), dict(sequences=-1), dict(max_q=-1), dict(max_k=-1), dict(q_rows=-1), dict(k_rows=-1), dict(q_rows=(1 << 30) + 1),
        dict(max_k=(1 << 30) + 1), dict(scale=NAN), dict(scale=INF), dict(cap=-1.0), dict(cap=NAN), dict(cap=INF), dict(causal=2), dict(causal=-1),
        dict(q_row=-512), dict(v_head=-64), dict(out_row=63), dict(out_head=0), dict(q_row=516), dict(k_head=4), dict(out_row=513), dict(q=None), dict(out=None),
        dict(q_offsets=None), dict(k_offsets=None), dict(k=None), dict(v=None), dict(q=PTR + 8), dict(v=PTR + 2), dict(lse=PTR + 2), dict(q_offsets=PTR + 1),
        dict(q_coords=PTR), dict(k_coords=PTR), dict(q_coords=PTR, k_coords=PTR), dict(q_coords=PTR + 4, k_coords=PTR, slopes=PTR),
        dict(dtype=vpe.VPE_F32, q_row=514))
] + [
    ("vpe_block_norm", norm_args, kw) for kw in (
        dict(dtype=3), dict(rows=-1), dict(requests=-1), dict(dim=0), dict(dim=8193), dict(post=3), dict(pre=-1), dict(eps=0.0), dict(eps=NAN), dict(eps=INF),
        dict(residual_scale=INF), dict(x=None), dict(out=None), dict(x_row=99), dict(out_row=0), dict(branch_row=99), dict(normed_row=-100),
        dict(out=PTR, out_row=104), dict(x=PTR + 2), dict(branch=PTR + 1), dict(dtype=vpe.VPE_F32, normed=PTR + 2), dict(gate=PTR + 3), dict(request=PTR + 2))
] + [
    ("vpe_adapter_linear", adapter_args, kw) for kw in (
        dict(dtype=9), dict(out_f32=2), dict(rows=-1), dict(in_features=0), dict(in_features=96), dict(out_features=0), dict(adapters=-1), dict(rank=0), dict(rank=12),
        dict(rank=136), dict(x=None), dict(weight=None), dict(out=None), dict(x_row=127), dict(x_row=132), dict(out_row=99), dict(x=PTR + 8), dict(weight=PTR + 2),
        dict(out=PTR + 1), dict(out_f32=1, out=PTR + 2), dict(bias=PTR + 2), dict(a=None), dict(b=None), dict(a=PTR + 8), dict(adapter=PTR + 2), dict(scale=PTR + 1),
        dict(workspace=None), dict(workspace_bytes=16), dict(workspace=PTR + 16), dict(rows=(1 << 30) + 1))
]


@pytest.mark.parametrize("call, make, kw", REFUSED, ids=lambda v: "-".join(f"{k}={x}" for k, x in v.items()) if isinstance(v, dict) else "")
def test_calls_that_are_refused(call, make, kw):
    args = make(**kw)
    assert getattr(vpe.lib(), call)(C.byref(args), None) == vpe.VPE_EINVAL
    assert vpe.vpe_last_error(None)


def test_null_arguments_are_refused():
    L = vpe.lib()
    for call in ("vpe_attention", "vpe_block_norm", "vpe_adapter_linear"):
        assert getattr(L, call)(None, None) == vpe.VPE_EINVAL
    n = C.c_uint64(0)
    for call, make in (("vpe_attention_workspace_bytes", attention_args), ("vpe_adapter_linear_workspace_bytes", adapter_args)):
        assert getattr(L, call)(None, C.byref(n)) == vpe.VPE_EINVAL
        assert getattr(L, call)(C.byref(make()), None) == vpe.VPE_EINVAL
        assert getattr(L, call)(C.byref(make()), C.byref(n)) == vpe.VPE_OK


@pytest.mark.parametrize("kw", [dict(sequences=0), dict(max_q=0), dict(q_rows=0)])
def test_attention_without_rows_enqueues_nothing(kw):
    # (no device here: a launch would fail)
    assert vpe.lib().vpe_attention(C.byref(attention_args(**kw, q=None, k=None, v=None, out=None, q_offsets=None, k_offsets=None)), None) == vpe.VPE_OK


def test_rows_of_length_zero_enqueue_nothing():
    assert vpe.lib().vpe_block_norm(C.byref(norm_args(rows=0, x=None, out=None)), None) == vpe.VPE_OK
    assert vpe.lib().vpe_adapter_linear(C.byref(adapter_args(rows=0, x=None, weight=None, out=None, workspace=None)), None) == vpe.VPE_OK


def test_workspace_of_attention_is_checked():
    """A few query rows against a long cache are split over the keys: partial results need a place."""
    a = attention_args(heads=8, kv_heads=8, sequences=1, max_q=1, q_rows=1, max_k=16384, k_rows=16384, k_row=512, v_row=512)
    n = C.c_uint64(0)
    assert vpe.lib().vpe_attention_workspace_bytes(C.byref(a), C.byref(n)) == vpe.VPE_OK
    if n.value:
        for kw in (dict(workspace=None), dict(workspace=PTR, workspace_bytes=n.value - 1), dict(workspace=PTR + 64, workspace_bytes=n.value)):
            for k, v in kw.items():
                setattr(a, k, v)
            assert vpe.lib().vpe_attention(C.byref(a), None) == vpe.VPE_EINVAL
    # the same sizes, the same workspace, whatever the pointers are
    b = attention_args(heads=8, kv_heads=8, sequences=1, max_q=1, q_rows=1, max_k=16384, k_rows=16384, q=None, k=None, lse=PTR)
    m = C.c_uint64(0)
    assert vpe.lib().vpe_attention_workspace_bytes(C.byref(b), C.byref(m)) == vpe.VPE_OK and m.value == n.value


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    f, i = torch.zeros, torch.int32
    off = torch.tensor([0, 4], dtype=i)
    q = f(4, 2, 64)

    def attend(**kw):
        base = dict(q=q, k=q, v=q, out=q.clone(), q_offsets=off, k_offsets=off, max_q=4, max_k=4)
        base.update(kw)
        vpe.attention(base.pop("q"), base.pop("k"), base.pop("v"), base.pop("out"), **base)

    bad = [lambda: attend(v=f(5, 2, 64)), lambda: attend(k=f(4, 2, 128)), lambda: attend(k=q.bfloat16(), v=q.bfloat16()), lambda: attend(q_offsets=off.long()),
           lambda: attend(k_offsets=off[:1]), lambda: attend(q=f(4, 64, 2).transpose(1, 2)), lambda: attend(slopes=f(3)), lambda: attend(lse=f(4, 3)),
           lambda: attend(prefix=off), lambda: attend(q_coords=f(4, 3), k_coords=f(4, 3), slopes=f(2)), lambda: attend(workspace=f(4)),
           lambda: attend(q=q.half(), k=q.half(), v=q.half(), out=q.half()),
           lambda: attend(),                                                             # (host memory)
           lambda: vpe.block_norm(f(3, 4), f(3, 5)), lambda: vpe.block_norm(f(3, 4), f(3, 4).bfloat16()),
           lambda: vpe.block_norm(f(3, 4), f(3, 4), branch=f(3, 4), normed=f(3, 4).bfloat16()), lambda: vpe.block_norm(f(3, 4), f(3, 4), gate=f(2, 4), scale=f(1, 4)),
           lambda: vpe.block_norm(f(3, 4), f(3, 4), post_gain=f(5)), lambda: vpe.block_norm(f(4, 3).t(), f(3, 4)), lambda: vpe.block_norm(f(3, 4), f(3, 4)),
           lambda: vpe.adapter_linear(f(3, 64), f(8, 128), f(3, 8)), lambda: vpe.adapter_linear(f(3, 64), f(8, 64), f(3, 9)),
           lambda: vpe.adapter_linear(f(3, 64), f(8, 64), f(3, 8).bfloat16()), lambda: vpe.adapter_linear(f(3, 64), f(8, 64), f(3, 8), a=f(1, 8, 64)),
           lambda: vpe.adapter_linear(f(3, 64), f(8, 64), f(3, 8), a=f(1, 8, 64), b=f(1, 9, 8), adapter=torch.zeros(3, dtype=i)),
           lambda: vpe.adapter_linear(f(3, 64), f(8, 64), f(3, 8))]
    for n, call in enumerate(bad):
        with pytest.raises(vpe.VpeError) as e:
            call()
        assert e.value.code == vpe.VPE_EINVAL, n
    # one row or one head: the stride of its axis says nothing
    assert binding._row_stride("x", torch.empty_strided((1, 8), (1, 1))) == 8


@pytest.mark.parametrize("over", [dict(max_q=2 ** 40), dict(max_k=2.5), dict(max_q=None), dict(cap=1e300), dict(cap="1")])
def test_sizes_that_are_no_numbers_of_their_fields_are_refused(over):
    import torch
    off, q = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(4, 2, 64)
    with pytest.raises(vpe.VpeError) as e:
        vpe.attention(q, q, q, q.clone(), q_offsets=off, k_offsets=off, **{**dict(max_q=4, max_k=4), **over})
    # (1e300 becomes an infinite float, which the library refuses: here the tensors' memory is refused before)
    assert e.value.code == vpe.VPE_EINVAL and ("device memory" not in str(e.value) or over.get("cap") == 1e300)


def test_rows_of_x_too_far_apart_for_a_tile_are_refused():
    a = adapter_args(x_row=(1 << 20) + 8)
    assert vpe.lib().vpe_adapter_linear(C.byref(a), None) == vpe.VPE_EINVAL and "stride" in vpe.vpe_last_error(None)
