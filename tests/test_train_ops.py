"""Lookup, grouped Update and distillation loss: refusals and workspace sizes (CPU), values and gradients against plain
float64 implementations (GPU).

Tolerances count roundings: a sum of K fp32 products or terms is off by at most K * 2^-23 of the sum of their magnitudes in any
order (2^-24 each where every addition rounds to nearest; the matrix instruction is given the factor 2), and an output by half a
step of its type, finfo(t).eps / 2 of the value.
"""
import ctypes
import itertools

import numpy as np
import pytest
import torch

from paper_2209_06800_amd import binding

DEV = "cuda:0"
gpu = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -23


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_within(got, ref, bound, what=""):
    """Elementwise; NaN where the reference has NaN and nowhere else, infinities equal."""
    got, ref, bound = got.detach().double().cpu(), ref.double().cpu(), bound.double().cpu()
    assert got.shape == ref.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN in other places"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), f"{what}: infinities"
    fine = ~(inf | torch.isnan(ref))
    err, bound = (got - ref)[fine].abs(), bound.expand_as(ref)[fine]
    bad = ~(err <= bound)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} values out of bound, worst {float((err / bound.clamp_min(1e-300)).max()):.3g} of it"


def strided(t, pad, lead=0):
    """The same values in a wider buffer of NaN (or -7 for ids), rows `pad` elements further apart, the first at element `lead`."""
    rows, cols = t.shape
    fill = float("nan") if t.is_floating_point() else -7
    buf = torch.full((rows * (cols + pad) + lead + 8,), fill, dtype=t.dtype, device=t.device)
    view = buf[lead: lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


# ---- refusals (CPU) ------------------------------------------------------------------------------------------
P = 0x100000            # an aligned address that no refused call touches


def embed_call(**kw):
    a = dict(n=4, it=1, ids=P, rows=10, tt=0, table=P, dim=8, ld=8, scale=1.0, ot=0, out=P, ldo=8)
    a.update(kw)
    return binding.lib().mgg_embed(a["n"], a["it"], a["ids"], a["rows"], a["tt"], a["table"], a["dim"], a["ld"], a["scale"], a["ot"], a["out"], a["ldo"], None)


def embed_grad_call(**kw):
    a = dict(n=4, it=1, ids=P, rows=10, gt=0, grad=P, dim=8, ld=8, scale=1.0, acc=0, ot=0, out=P, ldo=8, ws=P, bytes=1 << 20)
    a.update(kw)
    return binding.lib().mgg_embed_grad(a["n"], a["it"], a["ids"], a["rows"], a["gt"], a["grad"], a["dim"], a["ld"], a["scale"], a["acc"], a["ot"], a["out"],
                                        a["ldo"], a["ws"], a["bytes"], None)


def grouped_call(**kw):
    a = dict(n=4, g=2, ptr=P, at=0, a=P, lda=8, k=8, wt=0, w=P, bias=None, m=8, act=0, ot=0, out=P, ldo=8)
    a.update(kw)
    return binding.lib().mgg_update_grouped(a["n"], a["g"], a["ptr"], a["at"], a["a"], a["lda"], a["k"], a["wt"], a["w"], a["bias"], a["m"], a["act"], a["ot"],
                                            a["out"], a["ldo"], None)


def grouped_grad_call(**kw):
    a = dict(n=4, g=2, ptr=P, t=0, grad=P, ldg=8, act=0, ot=0, out=None, ldo=0, a=P, lda=8, k=8, w=P, m=8, dat=0, da=P, ldda=8, dwt=0, dw=P, db=None, acc=0,
             ws=P, bytes=1 << 24)
    a.update(kw)
    return binding.lib().mgg_update_grouped_grad(a["n"], a["g"], a["ptr"], a["t"], a["grad"], a["ldg"], a["act"], a["ot"], a["out"], a["ldo"], a["a"], a["lda"],
                                                 a["k"], a["w"], a["m"], a["dat"], a["da"], a["ldda"], a["dwt"], a["dw"], a["db"], a["acc"], a["ws"], a["bytes"],
                                                 None)


def distill_call(**kw):
    a = dict(n=4, c=8, zt=0, z=P, ldz=8, k=2, it=1, ids=P, ldi=2, tt=0, top=P, ldt=2, temp=1.0, w=None, loss=P, gt=0, grad=P, ldg=8, ws=P, bytes=1 << 24)
    a.update(kw)
    return binding.lib().mgg_distill_loss(a["n"], a["c"], a["zt"], a["z"], a["ldz"], a["k"], a["it"], a["ids"], a["ldi"], a["tt"], a["top"], a["ldt"], a["temp"],
                                          a["w"], a["loss"], a["gt"], a["grad"], a["ldg"], a["ws"], a["bytes"], None)


INVALID, UNSUPPORTED = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
REFUSALS = [
    (embed_call, INVALID, [dict(n=-1), dict(dim=0), dict(ld=7), dict(ldo=7), dict(rows=-1), dict(it=2), dict(tt=2), dict(ot=-1), dict(ids=None), dict(table=None),
                           dict(out=None), dict(ids=P + 4), dict(it=0, ids=P + 2), dict(table=P + 2), dict(tt=1, table=P + 1), dict(out=P + 2)]),
    (embed_call, UNSUPPORTED, [dict(rows=2 ** 31 - 1), dict(n=2 ** 31)]),
    (embed_grad_call, INVALID, [dict(n=-1), dict(dim=0), dict(ld=7), dict(ldo=7), dict(it=5), dict(gt=3), dict(ids=None), dict(grad=None), dict(out=None),
                                dict(acc=2), dict(ws=None), dict(ws=P + 128), dict(bytes=255), dict(ids=P + 4)]),
    (embed_grad_call, UNSUPPORTED, [dict(rows=2 ** 31 - 1), dict(n=2 ** 30 + 1)]),
    (grouped_call, INVALID, [dict(n=-1), dict(g=-1), dict(k=0), dict(m=0), dict(lda=7), dict(ldo=7), dict(ptr=None), dict(ptr=P + 4), dict(a=None), dict(w=None),
                             dict(out=None), dict(act=7), dict(at=2, wt=2), dict(ot=9), dict(a=P + 2), dict(bias=P + 2)]),
    (grouped_call, UNSUPPORTED, [dict(act=2), dict(wt=1), dict(at=1), dict(g=65536), dict(n=2 ** 31), dict(lda=2 ** 22 + 1), dict(k=2 ** 22 + 8, lda=2 ** 22 + 8)]),
    (grouped_grad_call, INVALID, [dict(n=-1), dict(g=-1), dict(k=0), dict(m=0), dict(ldg=7), dict(lda=7), dict(ldda=7), dict(ptr=None), dict(grad=None), dict(a=None),
                                  dict(w=None), dict(act=1), dict(act=1, out=P, ldo=7), dict(act=9), dict(acc=4), dict(t=2), dict(dat=2), dict(dwt=2), dict(ws=None),
                                  dict(ws=P + 16), dict(bytes=255), dict(db=P + 1), dict(dw=P + 2)]),
    (grouped_grad_call, UNSUPPORTED, [dict(act=2), dict(g=65536), dict(n=2 ** 31), dict(ldg=2 ** 22 + 1)]),
    (distill_call, INVALID, [dict(n=-1), dict(c=0), dict(k=0), dict(ldz=7), dict(ldi=1), dict(ldt=1), dict(ldg=7), dict(zt=2), dict(tt=2), dict(gt=2), dict(it=2),
                             dict(z=None), dict(ids=None), dict(top=None), dict(loss=None), dict(temp=0.0), dict(temp=-1.0), dict(temp=float("nan")),
                             dict(temp=float("inf")), dict(ws=None), dict(ws=P + 128), dict(bytes=255), dict(z=P + 2), dict(grad=P + 2, z=2 * P), dict(w=P + 2),
                             dict(z=P, grad=P, gt=1), dict(z=P, grad=P, ldg=9)]),
    (distill_call, UNSUPPORTED, [dict(k=1025, ldi=1025, ldt=1025), dict(n=2 ** 31 - 1), dict(c=2 ** 31 - 1, ldz=2 ** 31, ldg=2 ** 31)]),
]


@pytest.mark.parametrize("call,status,change", [(c, s, d) for c, s, ds in REFUSALS for d in ds], ids=lambda v: str(v) if isinstance(v, dict) else None)
def test_bad_arguments_are_refused(call, status, change):
    assert call(**change) == status
    assert len(binding.lib().mgg_last_error()) > 0


def test_calls_without_work_return_at_once():
    assert embed_call(n=0, ids=None, out=None) == binding.OK
    assert embed_grad_call(rows=0, out=None, grad=P) == binding.OK
    assert grouped_call(n=0, a=None, out=None) == binding.OK
    assert grouped_call(g=0, a=None, w=None, out=None) == binding.OK
    assert grouped_grad_call(g=0, w=None, a=None, da=None, dw=None) == binding.OK
    assert distill_call(n=0, z=None, ids=None, top=None, loss=None, grad=None) == binding.OK


def test_workspace_sizes():
    embed, grouped, distill = binding.mgg_embed_grad_workspace_bytes, binding.mgg_update_grouped_grad_workspace_bytes, binding.mgg_distill_workspace_bytes
    assert embed(-1, 10, 8) == 0 and embed(5, -1, 8) == 0 and embed(5, 10, 0) == 0 and embed(2 ** 30 + 1, 10, 8) == 0
    assert embed(0, 0, 1) > 0 and embed(1000, 10, 8) >= 1000 * 8
    assert grouped(-1, 1, 8, 8, F32) == 0 and grouped(1, 65536, 8, 8, F32) == 0 and grouped(1, 1, 0, 8, F32) == 0
    assert grouped(0, 0, 8, 8, F32) > 0
    assert grouped(100000, 4, 64, 64, BF16, act="relu") >= 100000 * 64 * 2          # the masked gradient
    assert distill(-1, 8) == 0 and distill(1, 0) == 0 and distill(0, 8) > 0
    # sizes beyond 32 bits are counted in 64
    assert grouped(2 ** 31 - 1, 1, 64, 4096, F32, act="relu") > 2 ** 40


def test_binding_refuses_what_the_c_abi_cannot_see():
    cpu = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        binding.mgg_embed(ids, cpu)
    with pytest.raises(TypeError):
        binding.mgg_embed(ids.short(), cpu)
    with pytest.raises(ValueError):
        binding.mgg_embed(torch.zeros(4, 2, dtype=torch.int64), cpu)
    with pytest.raises(ValueError):
        binding.mgg_embed(torch.zeros(8, dtype=torch.int64)[::2], cpu)
    with pytest.raises(ValueError):
        binding.mgg_embed_grad(ids, torch.zeros(5, 8), 10)
    ptr = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        binding.mgg_update_grouped(ptr.int(), cpu, torch.zeros(2, 8, 8))
    with pytest.raises(ValueError):
        binding.mgg_update_grouped(ptr, cpu, torch.zeros(3, 8, 8))
    with pytest.raises(ValueError):
        binding.mgg_update_grouped(ptr, cpu, torch.zeros(2, 7, 8))
    with pytest.raises(ValueError):
        binding.mgg_update_grouped(ptr, cpu, torch.zeros(2, 8, 8), torch.zeros(2, 7))
    with pytest.raises(ValueError):
        binding.mgg_update_grouped_grad(ptr, cpu, cpu, torch.zeros(2, 8, 8), "relu")
    with pytest.raises(binding.MggError) as e:
        binding.mgg_update_grouped_grad(ptr, cpu.bfloat16(), cpu, torch.zeros(2, 8, 8))
    assert e.value.status == UNSUPPORTED
    with pytest.raises(ValueError):
        binding.mgg_distill_loss(cpu, torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 3))
    with pytest.raises(TypeError):
        binding.mgg_distill_loss(cpu, torch.zeros(4, 2, dtype=torch.int16), torch.zeros(4, 2))
    with pytest.raises(ValueError):
        binding.mgg_distill_loss(cpu, torch.zeros(4, 2, dtype=torch.int64), torch.zeros(4, 2), row_weight=torch.zeros(3))


# ---- lookup --------------------------------------------------------------------------------------------------
def draw_ids(n, rows, seed, skew=2.0, bad=0.1):
    rng = np.random.default_rng(seed)
    ids = np.minimum((rng.random(n) ** skew * rows).astype(np.int64), max(rows - 1, 0))
    out = rng.random(n) < bad
    ids[out] = rng.choice([-1, rows, rows + 5, -(2 ** 31), 2 ** 31 - 1], size=n)[out]
    return torch.from_numpy(ids)


@gpu
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (1, 7, 4096), (5, 300, 7), (64, 2, 8), (257, 1000, 95), (1000, 33, 64), (3, 50, 2051), (70001, 513, 24), (20000, 100, 602)])
@pytest.mark.parametrize("tin,tout", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
def test_embed_copies_scaled_rows(n, rows, dim, tin, tout):
    g = torch.Generator().manual_seed(n + rows + dim)
    table = torch.randn(rows, dim, generator=g).to(tin)
    for it, scale, pad, lead in ((torch.int64, 1.0, 0, 0), (torch.int32, 3.7, 3, 1)):
        ids = draw_ids(n, rows, n + dim).to(it)
        there = (ids >= 0) & (ids < rows)
        ref = torch.where(there[:, None], table[ids.clamp(0, rows - 1).long()].float() * torch.tensor(scale), torch.zeros(())).to(tout)
        out = strided(torch.zeros(n, dim, dtype=tout, device=DEV), pad, lead)
        got = binding.mgg_embed(ids.to(DEV), strided(table.to(DEV), pad, lead), scale=scale, out=out)
        assert got is out
        assert torch.equal(got.cpu(), ref)
        whole = out._base
        assert int(torch.isnan(whole).sum()) == whole.numel() - n * dim         # nothing beside the rows was written


def table_grad(ids, grad, rows, scale, into=None):
    there = (ids >= 0) & (ids < rows)
    ref = torch.zeros(rows, grad.shape[1], dtype=torch.float64)
    mag, count = torch.zeros_like(ref), torch.zeros(rows, dtype=torch.float64)
    at, g = ids[there].long(), grad[there].double() * scale
    ref.index_add_(0, at, g)
    mag.index_add_(0, at, g.abs())
    count.index_add_(0, at, torch.ones(at.numel(), dtype=torch.float64))
    if into is not None:
        ref, mag = ref + into.double(), mag + into.double().abs()
    return ref, mag, count


@gpu
@pytest.mark.parametrize("n,rows,dim", [(0, 5, 8), (1, 1, 1), (1, 300, 130), (2, 257, 64), (63, 3, 7), (64, 70000, 20), (65, 4, 256), (1000, 5003, 95), (4096, 256, 33),
                                        (4097, 255, 16), (9000, 40, 602), (20011, 65536, 8), (50000, 1, 24), (100003, 700, 65), (33000, 300000, 4), (600001, 3000, 8), (8192, 100000, 16), (8193, 1 << 20, 8)])
@pytest.mark.parametrize("tin,tout", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
def test_embed_grad_sums_by_id(n, rows, dim, tin, tout):
    g = torch.Generator().manual_seed(3 * n + rows + dim)
    grad = torch.randn(n, dim, generator=g).to(tin)
    ids = draw_ids(n, rows, n + dim, bad=0.05)
    for it, accumulate, pad, lead in ((torch.int64, False, 0, 0), (torch.int32, True, 3, 1)):
        scale = 0.75 if accumulate else 2.5
        into = torch.randn(rows, dim, generator=g).to(tout) if accumulate else None
        ref, mag, count = table_grad(ids, grad, rows, scale, into)
        out = strided((into if accumulate else torch.full((rows, dim), 9.0, dtype=tout)).to(DEV), pad, lead)
        args = (ids.to(it).to(DEV), strided(grad.to(DEV), pad, lead) if n else grad.to(DEV), rows)
        got = binding.mgg_embed_grad(*args, scale=scale, out=out, accumulate=accumulate)
        assert_within(got, ref, (count[:, None] + 3) * U * mag + half_step(tout) * ref.abs(), f"{it} accumulate {accumulate}")
        if accumulate:
            assert torch.equal(got.cpu()[count == 0], into[count == 0])
        else:
            assert torch.equal(binding.mgg_embed_grad(*args, scale=scale, out_dtype=tout), got)      # the same bits again
        whole = out._base
        assert int(torch.isnan(whole).sum()) == whole.numel() - rows * dim


@gpu
def test_embed_grad_with_every_id_outside():
    ids = torch.full((500,), -1, dtype=torch.int64, device=DEV)
    grad = torch.full((500, 12), float("nan"), device=DEV)
    assert torch.equal(binding.mgg_embed_grad(ids, grad, 9), torch.zeros(9, 12, device=DEV))
    kept = torch.ones(9, 12, device=DEV)
    assert torch.equal(binding.mgg_embed_grad(ids, grad, 9, out=kept.clone(), accumulate=True), kept)


@gpu
def test_tables_and_gradients_beyond_32_bit_offsets():
    rows, dim = 1100000, 4096                   # 9 GB of bf16, the last rows at offsets past 2^32 elements
    table = torch.zeros(rows, dim, dtype=BF16, device=DEV)
    ids = torch.tensor([rows - 1, 0, rows - 1, 524288, 1048577], device=DEV)
    table[ids] = torch.arange(5, device=DEV, dtype=BF16)[:, None]
    want = table[ids].clone()
    assert torch.equal(binding.mgg_embed(ids, table), want)
    grad = torch.ones(5, dim, device=DEV)
    binding.mgg_embed_grad(ids, grad, rows, out=table)
    assert torch.equal(table[ids].float(), torch.tensor([2.0, 1.0, 2.0, 1.0, 1.0], device=DEV)[:, None].expand(5, dim))
    assert float(table.sum(dtype=torch.float32)) == 5 * dim


# ---- grouped Update ------------------------------------------------------------------------------------------
def group_ptr(counts, before=0):
    return torch.tensor(np.concatenate([[before], before + np.cumsum(counts)]), dtype=torch.int64)


def grouped_reference(ptr, a, w, bias, act):
    n, groups = a.shape[0], w.shape[0]
    ref = torch.full((n, w.shape[2]), float("nan"), dtype=torch.float64)
    mag = torch.zeros_like(ref)
    for g in range(groups):
        lo, hi = int(ptr[g]), int(ptr[g + 1])
        ref[lo:hi] = a[lo:hi].double() @ w[g].double()
        mag[lo:hi] = a[lo:hi].double().abs() @ w[g].double().abs()
        if bias is not None:
            ref[lo:hi] += bias[g].double()
            mag[lo:hi] += bias[g].double().abs()
    return (torch.relu(ref) if act == "relu" else ref), mag


GROUPED = [
    # counts, d_in, d_out
    ([1], 1, 1), ([0, 1, 0], 5, 3), ([3, 0, 130, 1, 64], 64, 64), ([200], 128, 256), ([127, 129], 100, 256), ([5, 0, 0, 40], 602, 47), ([33, 31, 0, 2], 47, 130),
    ([300, 1, 77], 256, 384), ([1] * 70 + [0] * 30 + [9] * 40, 72, 40), ([16, 0, 17, 15], 520, 136), ([700, 20], 65, 63), ([2, 2], 7, 1000), ([520], 192, 264),
    ([1, 2, 0, 1], 1030, 200),
]


@gpu
@pytest.mark.parametrize("counts,d_in,d_out", GROUPED)
@pytest.mark.parametrize("dtype,tout,act,with_bias", [(BF16, BF16, "relu", True), (BF16, F32, "none", False), (F32, F32, "relu", True), (F32, BF16, "none", True)])
def test_grouped_update(counts, d_in, d_out, dtype, tout, act, with_bias):
    g = torch.Generator().manual_seed(sum(counts) + d_in + d_out)
    n, groups = sum(counts), len(counts)
    a = torch.randn(n, d_in, generator=g).to(dtype)
    w = (torch.randn(groups, d_in, d_out, generator=g) * d_in ** -0.5).to(dtype)
    bias = torch.randn(groups, d_out, generator=g) if with_bias else None
    ptr = group_ptr(counts)
    ref, mag = grouped_reference(ptr, a, w, bias, act)
    for pad, lead in ((0, 0), (8, 0), (5, 1)):
        out = strided(torch.zeros(n, d_out, dtype=tout, device=DEV), pad, lead)
        got = binding.mgg_update_grouped(ptr.to(DEV), strided(a.to(DEV), pad, lead), w.to(DEV), None if bias is None else bias.to(DEV), act, out=out)
        assert_within(got, ref, (d_in + 2) * U * mag + half_step(tout) * ref.abs(), f"pad {pad} lead {lead}")
        whole = out._base
        assert int(torch.isnan(whole).sum()) == whole.numel() - n * d_out


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_grouped_rows_outside_the_groups_are_left_alone(dtype):
    n, d_in, d_out = 500, 40, 72
    ptr = torch.tensor([100, 230, 230, 400], device=DEV)
    a = torch.full((n, d_in), float("nan"), dtype=dtype, device=DEV)       # rows of no group may hold anything
    a[100:400] = torch.randn(300, d_in, device=DEV).to(dtype)
    w = torch.randn(3, d_in, d_out, device=DEV).to(dtype)
    w[1] = float("nan")                                                     # a group without rows
    out = torch.full((n, d_out), 7.0, dtype=dtype, device=DEV)
    binding.mgg_update_grouped(ptr, a, w, out=out)
    assert bool((out[:100] == 7).all()) and bool((out[400:] == 7).all()) and not bool(torch.isnan(out).any())
    dz = torch.full((n, d_out), float("nan"), dtype=dtype, device=DEV)
    dz[100:400] = torch.randn(300, d_out, device=DEV).to(dtype)
    da = torch.full((n, d_in), 7.0, dtype=dtype, device=DEV)
    got = binding.mgg_update_grouped_grad(ptr, dz, a, w, grad_a=da, need_bias=True)
    assert bool((da[:100] == 7).all()) and bool((da[400:] == 7).all())
    assert all(not bool(torch.isnan(t).any()) for t in got)
    assert not bool(got[1][1].any()) and not bool(got[2][1].any())


@gpu
@pytest.mark.parametrize("offsets", [[-5, 20, 90], [0, 60, 1000], [50, 20, 40], [0, 2 ** 40, 64], [64, 64, 64]])
def test_grouped_offsets_out_of_range_stay_inside_the_buffers(offsets):
    """What such offsets compute is not defined where groups overlap; the buffers around the matrices stay as they were."""
    n, d = 64, 24
    ptr = torch.tensor(offsets, device=DEV)
    around = torch.full((3 * n, d), 5.0, device=DEV)
    binding.mgg_update_grouped(ptr, torch.ones(n, d, device=DEV), torch.ones(2, d, d, device=DEV), out=around[n:2 * n])
    assert bool((around[:n] == 5).all()) and bool((around[2 * n:] == 5).all())
    da, dw, db = binding.mgg_update_grouped_grad(ptr, torch.ones(n, d, device=DEV), torch.ones(n, d, device=DEV), torch.ones(2, d, d, device=DEV),
                                                 grad_a=around[n:2 * n], need_bias=True)
    assert bool((around[:n] == 5).all()) and bool((around[2 * n:] == 5).all())
    assert bool((dw <= n).all()) and bool((db <= n).all())


def grouped_grad_reference(ptr, dz, a, w):
    n, groups = a.shape[0], w.shape[0]
    da = torch.full(a.shape, float("nan"), dtype=torch.float64)
    dw, db = torch.zeros(w.shape, dtype=torch.float64), torch.zeros(groups, w.shape[2], dtype=torch.float64)
    mags = [torch.zeros_like(da), torch.zeros_like(dw), torch.zeros_like(db)]
    for g in range(groups):
        lo, hi = int(ptr[g]), int(ptr[g + 1])
        z, x, m = dz[lo:hi].double(), a[lo:hi].double(), w[g].double()
        da[lo:hi], dw[g], db[g] = z @ m.t(), x.t() @ z, z.sum(0)
        mags[0][lo:hi], mags[1][g], mags[2][g] = z.abs() @ m.abs().t(), x.abs().t() @ z.abs(), z.abs().sum(0)
    return (da, dw, db), mags


@gpu
@pytest.mark.parametrize("counts,d_in,d_out", GROUPED + [([2000, 3, 900], 40, 24), ([5000], 16, 16)])
@pytest.mark.parametrize("dtype,tw,act,accumulate", [(BF16, F32, "relu", False), (BF16, BF16, "none", True), (F32, F32, "none", False), (F32, F32, "relu", True)])
def test_grouped_gradients(counts, d_in, d_out, dtype, tw, act, accumulate):
    g = torch.Generator().manual_seed(sum(counts) + 2 * d_in + d_out)
    n, groups = sum(counts), len(counts)
    a = torch.randn(n, d_in, generator=g).to(dtype)
    w = (torch.randn(groups, d_in, d_out, generator=g) * d_in ** -0.5).to(dtype)
    dout = torch.randn(n, d_out, generator=g).to(dtype)
    ptr = group_ptr(counts)
    out = torch.relu(torch.randn(n, d_out, generator=g)).to(dtype) if act == "relu" else None
    dz = dout if out is None else torch.where(out > 0, dout, torch.zeros((), dtype=dtype))
    refs, mags = grouped_grad_reference(ptr, dz, a, w)
    into = torch.randn(w.shape, generator=g).to(tw) if accumulate else None
    into_b = torch.randn(groups, d_out, generator=g) if accumulate else None
    if accumulate:
        refs = (refs[0], refs[1] + into.double(), refs[2] + into_b.double())
        mags = (mags[0], mags[1] + into.double().abs(), mags[2] + into_b.double().abs())
    longest = max(counts)
    terms = (d_out + 2, longest + 3, longest + 3)
    for pad, lead in ((0, 0), (8, 0), (5, 1)):
        dev = [strided(t.to(DEV), pad, lead) for t in (dout, a)] + [None if out is None else strided(out.to(DEV), pad, lead)]
        da = strided(torch.zeros(n, d_in, dtype=dtype, device=DEV), pad, lead)
        def call():
            return binding.mgg_update_grouped_grad(ptr.to(DEV), dev[0], dev[1], w.to(DEV), act, out=dev[2], need_bias=True, grad_a=da,
                                                   grad_w=None if into is None else into.to(DEV), grad_bias=None if into_b is None else into_b.to(DEV),
                                                   w_grad_dtype=tw, accumulate=accumulate)
        got = call()
        for name, x, ref, mag, k, t in zip(("grad_a", "grad_w", "grad_bias"), got, refs, mags, terms, (dtype, tw, F32)):
            assert_within(x, ref, k * U * mag + half_step(t) * ref.abs(), f"{name}, pad {pad} lead {lead}")
        whole = da._base
        assert int(torch.isnan(whole).sum()) == whole.numel() - n * d_in
        first = [t.clone() for t in got]
        assert all(torch.equal(x, y) for x, y in zip(first, call()))          # the same bits again


# Sizes at which the kernels for many rows run: (counts, d_in, d_out, dtype).  Ends inside tiles and inside 16 bytes, empty groups, groups
# shorter than a tile beside long ones.
MANY = [
    ([4000, 0, 1, 4700, 299], 200, 2048, BF16),         # whole chunks: large tiles forward; medium ones of the weights' gradient
    ([4000, 0, 1, 4700, 299], 2048, 200, BF16),         # large tiles of the rows' gradient
    ([64] * 9 + [0, 130, 3] + [70] * 8, 1024, 1032, BF16),       # large tiles of the weights' gradient, up to three steps
    ([2500, 7, 2493], 203, 1001, BF16),
    ([2500, 7, 2493], 1001, 203, BF16),
    ([12000, 1, 8000], 130, 47, BF16),
    ([12000, 1, 8000], 48, 136, BF16),
    ([5000, 0, 4001], 101, 300, F32),
    ([5000, 0, 4001], 300, 101, F32),
    ([3000, 200, 2800], 64, 64, BF16),
    ([257] * 40, 512, 40, F32),
    ([9000, 1, 8001], 56, 40, BF16),
    ([9000, 1, 8001], 47, 33, BF16),
    ([5000, 0, 4001], 100, 300, F32),
]


@gpu
@pytest.mark.parametrize("counts,d_in,d_out,dtype", MANY)
def test_grouped_update_and_gradients_of_many_rows(counts, d_in, d_out, dtype):
    g = torch.Generator().manual_seed(sum(counts) + d_in + 3 * d_out)
    n, groups = sum(counts), len(counts)
    a = torch.randn(n, d_in, generator=g).to(dtype)
    w = (torch.randn(groups, d_in, d_out, generator=g) * d_in ** -0.5).to(dtype)
    bias, dz = torch.randn(groups, d_out, generator=g), torch.randn(n, d_out, generator=g).to(dtype)
    ptr = group_ptr(counts)
    ref, mag = grouped_reference(ptr, a, w, bias, "relu")
    out = strided(torch.zeros(n, d_out, dtype=dtype, device=DEV), 3, 1)
    args = (ptr.to(DEV), a.to(DEV), w.to(DEV), bias.to(DEV), "relu")
    got = binding.mgg_update_grouped(*args, out=out)
    assert_within(got, ref, (d_in + 2) * U * mag + half_step(dtype) * ref.abs(), "out")
    assert int(torch.isnan(out._base).sum()) == out._base.numel() - n * d_out
    assert torch.equal(binding.mgg_update_grouped(*args), got)
    masked = torch.where(got.cpu() > 0, dz, torch.zeros((), dtype=dtype))
    refs, mags = grouped_grad_reference(ptr, masked, a, w)
    def call():
        return binding.mgg_update_grouped_grad(args[0], dz.to(DEV), args[1], args[2], "relu", out=got, need_bias=True)
    grads = call()
    for name, x, r, m, k in zip(("grad_a", "grad_w", "grad_bias"), grads, refs, mags, (d_out + 2, max(counts) + 3, max(counts) + 3)):
        assert_within(x, r, k * U * m + half_step(x.dtype) * r.abs(), name)
    assert all(torch.equal(x, y) for x, y in zip(grads, call()))


@gpu
def test_grouped_gradients_one_at_a_time():
    counts, d_in, d_out = [70, 0, 130], 48, 56
    ptr = group_ptr(counts).to(DEV)
    a, dz, w = torch.randn(200, d_in, device=DEV), torch.randn(200, d_out, device=DEV), torch.randn(3, d_in, d_out, device=DEV)
    out = torch.randn(200, d_out, device=DEV)
    for act, o in (("none", None), ("relu", out)):
        both = binding.mgg_update_grouped_grad(ptr, dz, a, w, act, out=o, need_bias=True)
        only_a = binding.mgg_update_grouped_grad(ptr, dz, a, w, act, out=o, need_w=False)
        only_w = binding.mgg_update_grouped_grad(ptr, dz, a, w, act, out=o, need_a=False)
        only_b = binding.mgg_update_grouped_grad(ptr, dz, a, w, act, out=o, need_a=False, need_w=False, need_bias=True)
        assert only_a[1] is None and only_w[0] is None and only_b[:2] == (None, None)
        assert torch.equal(only_a[0], both[0]) and torch.equal(only_w[1], both[1]) and torch.equal(only_b[2], both[2])


@gpu
def test_grouped_infinities_and_nan_stay_in_their_row_and_column():
    n, d_in, d_out = 150, 70, 90
    for dtype in (F32, BF16):
        a, w = torch.randn(n, d_in, device=DEV).to(dtype), torch.randn(1, d_in, d_out, device=DEV).to(dtype)
        ptr = torch.tensor([0, n], device=DEV)
        a[3, 5], a[149, 69], w[0, 69, 89] = float("inf"), float("nan"), float("nan")
        bad = ~torch.isfinite(binding.mgg_update_grouped(ptr, a, w, out_dtype=F32))
        want = torch.zeros(n, d_out, dtype=torch.bool, device=DEV)
        want[3], want[149], want[:, 89] = True, True, True
        assert torch.equal(bad, want)
        # a ReLU's mask is by the forward output: what the gradient holds at masked places is not read into the sums
        out = torch.ones(n, d_out, device=DEV).to(dtype)
        out[:, 7] = 0
        dz = torch.randn(n, d_out, device=DEV).to(dtype)
        dz[:, 7] = float("nan")
        x = torch.randn(n, d_in, device=DEV).to(dtype)
        got = binding.mgg_update_grouped_grad(ptr, dz, x, torch.ones(1, d_in, d_out, device=DEV, dtype=dtype), "relu", out=out, need_bias=True)
        assert all(bool(torch.isfinite(t).all()) for t in got)
        assert not bool(got[1][0, :, 7].any()) and not bool(got[2][0, 7].any())


# ---- distillation --------------------------------------------------------------------------------------------
def distill_reference(z, ids, top, temperature, weight):
    """Row by row, in float64: loss, gradient, and the sums of magnitudes that the bounds need."""
    n, classes = z.shape
    t = float(np.float32(temperature))
    loss, grad = torch.zeros(n, dtype=torch.float64), torch.zeros(n, classes, dtype=torch.float64)
    loss_mag, grad_mag = torch.zeros_like(loss), torch.zeros_like(grad)
    for r in range(n):
        w = float(weight[r]) if weight is not None else 1.0
        keep = [(int(i), float(x) / t) for i, x in zip(ids[r], top[r]) if 0 <= int(i) < classes]
        x = z[r].double() / t
        if w == 0.0 or not keep or all(v == -np.inf for _, v in keep) or bool((x == -np.inf).all()):
            continue
        v = torch.tensor([v for _, v in keep], dtype=torch.float64)
        log_p, log_q = torch.log_softmax(v, 0), torch.log_softmax(x, 0)
        at = torch.tensor([i for i, _ in keep])
        p = log_p.exp()
        some = p != 0
        diff = (log_p - log_q[at])[some]
        loss[r] = w * t * t * (p[some] * diff).sum()
        q = log_q.exp()
        mass = torch.zeros(classes, dtype=torch.float64).index_add_(0, at, p)
        grad[r] = w * t * (q - mass)
        finite = x[torch.isfinite(x)]
        spread = float((finite.max() - finite).max()) + float(finite.abs().max()) if finite.numel() else 0.0
        tv = v[torch.isfinite(v)]
        spread_p = float((tv.max() - tv).max()) + float(tv.abs().max()) if tv.numel() else 0.0
        # exponents off by a few roundings of numbers up to `spread`, exp and log by two more, sums of up to classes / 64 terms a lane
        e = (4 * spread + 4 * spread_p + classes / 64 + len(keep) + 40) * U
        loss_mag[r] = abs(w) * t * t * (float((p[some] * (diff.abs() + 2)).sum()) * e)
        grad_mag[r] = abs(w) * t * (q + mass) * e
    return loss, grad, loss_mag, grad_mag


def draw_distill(n, classes, k, seed, tz, tt, missing=0.1):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.normal(0, 3, (n, classes)).astype(np.float32)).to(tz)
    ids = torch.from_numpy(np.stack([rng.permutation(classes)[:k] if k <= classes else rng.integers(0, classes, k) for _ in range(n)]).reshape(n, k)).long()
    ids[torch.from_numpy(rng.random((n, k)) < missing)] = -1
    top = torch.from_numpy(rng.normal(2, 3, (n, k)).astype(np.float32)).to(tt)
    weight = torch.from_numpy((rng.random(n) * (rng.random(n) > 0.2)).astype(np.float32))
    return z, ids, top, weight


@gpu
@pytest.mark.parametrize("n,classes,k", [(1, 1, 1), (3, 2, 5), (300, 7, 3), (1000, 47, 8), (65, 64, 1), (20, 129, 40), (9, 1000, 64), (5, 4099, 200), (2, 50021, 20),
                                         (1, 200003, 64), (40, 8200, 16), (3, 33000, 1024), (600, 2051, 4), (129, 20001, 7), (128, 70001, 9), (150, 9001, 3)])
@pytest.mark.parametrize("tz,tt,tg", [(F32, F32, F32), (BF16, F32, BF16), (BF16, BF16, F32), (F32, BF16, BF16)])
def test_distill_loss_and_gradient(n, classes, k, tz, tt, tg):
    z, ids, top, weight = draw_distill(n, classes, k, n + classes + k, tz, tt)
    for it, temperature, w, pad, lead in ((torch.int64, 2.0, weight, 0, 0), (torch.int32, 0.7, None, 3, 1)):
        loss, grad, loss_bound, grad_bound = distill_reference(z, ids, top, temperature, w)
        dz, di, dt = strided(z.to(DEV), pad, lead), strided(ids.to(it).to(DEV), pad, lead), strided(top.to(DEV), pad, lead)
        dw = None if w is None else w.to(DEV)
        out = strided(torch.zeros(n, classes, dtype=tg, device=DEV), pad, lead)
        got, got_grad = binding.mgg_distill_loss(dz, di, dt, temperature=temperature, row_weight=dw, grad=out)
        assert_within(got, loss, loss_bound + half_step(F32) * loss.abs(), "loss")
        assert_within(got_grad, grad, grad_bound + half_step(tg) * grad.abs() + 1e-37, "gradient")
        whole = out._base
        assert int(torch.isnan(whole).sum()) == whole.numel() - n * classes
        alone = binding.mgg_distill_loss(dz, di, dt, temperature=temperature, row_weight=dw)
        assert_within(alone, loss, loss_bound + half_step(F32) * loss.abs(), "loss alone")
        again, again_grad = binding.mgg_distill_loss(dz, di, dt, temperature=temperature, row_weight=dw, need_grad=True, grad_dtype=tg)
        assert torch.equal(again, got) and torch.equal(again_grad, got_grad)


@gpu
@pytest.mark.parametrize("classes", [47, 3000, 150000])
@pytest.mark.parametrize("tz", [F32, BF16])
def test_distill_rows_that_masks_leave_empty(classes, tz):
    inf, nan, low = float("inf"), float("nan"), float(torch.finfo(tz).min)
    n, k = 12, 4
    z, ids, top, _ = draw_distill(n, classes, k, classes, tz, F32, missing=0.0)
    weight = torch.ones(n)
    z[0] = -inf                                             # nothing left to choose
    z[1], weight[1] = nan, 0.0                              # a row that is not looked at
    ids[2], top[2] = -1, nan                                # no teacher
    top[3] = -inf                                           # a teacher with no mass
    z[4] = low                                              # masked by the lowest value: equal chances
    z[5, 1:] = -inf                                         # one class left
    ids[5] = torch.tensor([0, -1, -1, -1])
    z[6, ids[6, 1]] = -inf                                  # the teacher gives p > 0 to a class the student cannot have
    z[7, ids[7, 2]], top[7, 2] = -inf, -inf                 # ... and p = 0
    ids[8, 1], top[8, 1] = classes, nan                     # an entry outside the classes
    ids[9] = ids[9, 0]                                      # one class four times
    z[10, 0] = nan
    z[11, classes // 2:], ids[11] = low, torch.arange(4)
    loss, grad, loss_bound, grad_bound = distill_reference(z, ids, top, 1.5, weight)
    loss_bound[4], grad_bound[4] = 2e-6 * (1 + loss[4].abs()) * (classes / 64 + 40), 1e-6 * grad[4].abs() * (classes / 64 + 40)      # (equal logits: no spread)
    loss_bound[11], grad_bound[11] = 2e-6 * (1 + loss[11].abs()) * (classes / 64 + 40), 2e-6 * (grad[11].abs() + 1e-6) * (classes / 64 + 40)
    got, got_grad = binding.mgg_distill_loss(z.to(DEV), ids.to(DEV), top.to(DEV), temperature=1.5, row_weight=weight.to(DEV), need_grad=True, grad_dtype=F32)
    for r in (0, 1, 2, 3):
        assert float(got[r]) == 0.0 and not bool(got_grad[r].any())
    assert_within(got, loss, loss_bound + half_step(F32) * loss.abs() + 1e-30, "loss")
    assert_within(got_grad, grad, grad_bound + half_step(F32) * grad.abs() + 1e-30, "gradient")


@gpu
@pytest.mark.parametrize("n,classes", [(300, 47), (64, 3001), (2, 140000)])
@pytest.mark.parametrize("tz", [F32, BF16])
def test_distill_gradient_in_place_of_the_logits(n, classes, tz):
    z, ids, top, weight = (t.to(DEV) for t in draw_distill(n, classes, 6, classes, tz, F32))
    want, want_grad = binding.mgg_distill_loss(z, ids, top, temperature=2.0, row_weight=weight, need_grad=True)
    got, got_grad = binding.mgg_distill_loss(z, ids, top, temperature=2.0, row_weight=weight, grad=z)
    assert got_grad is z and torch.equal(got, want) and torch.equal(got_grad, want_grad)


@gpu
def test_distill_gradient_against_differences():
    """(loss(z + h) - loss(z - h)) / 2h in float64, from the reference whose loss the kernel's equals."""
    n, classes, k, h = 4, 23, 5, 1e-5
    z, ids, top, weight = draw_distill(n, classes, k, 5, F32, F32)
    weight += 0.5
    _, grad = binding.mgg_distill_loss(z.to(DEV), ids.to(DEV), top.to(DEV), temperature=1.7, row_weight=weight.to(DEV), need_grad=True)
    for r, c in itertools.product(range(n), range(0, classes, 3)):
        up, down = z.double().clone(), z.double().clone()
        up[r, c] += h
        down[r, c] -= h
        slope = (distill_reference(up, ids, top, 1.7, weight)[0][r] - distill_reference(down, ids, top, 1.7, weight)[0][r]) / (2 * h)
        # the difference quotient: third derivatives (below 4 here) times h^2, and 2^-52 of losses below 100 over h
        assert abs(float(grad[r, c]) - float(slope)) < 1e-5 * abs(float(slope)) + 1e-6


# ---- together ------------------------------------------------------------------------------------------------
def step(ids, table, ptr, order, w1, b1, w2, top_ids, top, weight, scale=2.0, temperature=2.0):
    """Tokens -> rows in the order of their experts -> the experts' layer -> logits -> loss, and all gradients back."""
    x = binding.mgg_embed(ids[order], table, scale=scale)
    hidden = binding.mgg_update_grouped(ptr, x, w1, b1, "relu")
    logits = binding.mgg_update(hidden, w2)
    loss, dlogits = binding.mgg_distill_loss(logits, top_ids, top, temperature=temperature, row_weight=weight, need_grad=True)
    whole = torch.tensor([0, x.shape[0]], device=x.device) if not torch.cuda.is_current_stream_capturing() else WHOLE[x.shape[0]]
    dhidden, dw2 = binding.mgg_update_grouped_grad(whole, dlogits, hidden, w2[None])
    dx, dw1, db1 = binding.mgg_update_grouped_grad(ptr, dhidden, x, w1, "relu", out=hidden, need_bias=True)
    dtable = binding.mgg_embed_grad(ids[order], dx, table.shape[0], scale=scale)
    return loss, dtable, dw1, db1, dw2[0]


WHOLE = {}


def step_inputs(seed):
    g = torch.Generator().manual_seed(seed)
    n, rows, dim, hid, classes, groups, k = 700, 300, 48, 72, 47, 5, 6
    ids = torch.randint(0, rows, (n,), generator=g)
    expert = torch.randint(0, groups - 1, (n,), generator=g)            # the last one has no row
    order = torch.argsort(expert, stable=True)
    counts = torch.bincount(expert, minlength=groups)
    ptr = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    table = torch.randn(rows, dim, generator=g)
    w1, b1 = torch.randn(groups, dim, hid, generator=g) * dim ** -0.5, torch.randn(groups, hid, generator=g) * 0.1
    w2 = torch.randn(hid, classes, generator=g) * hid ** -0.5
    top_ids = torch.stack([torch.randperm(classes, generator=g)[:k] for _ in range(n)])
    top = torch.randn(n, k, generator=g) * 2
    weight = torch.rand(n, generator=g) / n
    return ids, table, ptr, order, w1, b1, w2, top_ids, top, weight


def step_reference(ids, table, ptr, order, w1, b1, w2, top_ids, top, weight, scale=2.0, t=2.0):
    leaves = [x.double().requires_grad_() for x in (table, w1, b1, w2)]
    x = leaves[0][ids[order]] * scale
    hidden = torch.cat([torch.relu(x[int(ptr[g]):int(ptr[g + 1])] @ leaves[1][g] + leaves[2][g]) for g in range(w1.shape[0])])
    log_q = torch.log_softmax(hidden @ leaves[3] / t, 1)
    log_p = torch.log_softmax(top.double() / t, 1)
    loss = weight.double() * t * t * (log_p.exp() * (log_p - log_q.gather(1, top_ids))).sum(1)
    loss.sum().backward()
    return [loss.detach()] + [leaf.grad for leaf in leaves]


@gpu
def test_a_training_step():
    """Against autograd in float64.  fp32 throughout: five products and sums of at most 300 terms one after the other, 2-norms within
    5 * 300 * 2^-23."""
    args = step_inputs(1)
    got = step(*(t.to(DEV) for t in args))
    for name, x, ref in zip(("loss", "table", "w1", "b1", "w2"), got, step_reference(*args)):
        rel = float((x.double().cpu() - ref).norm() / ref.norm())
        assert rel < 5 * 300 * U, (name, rel)


@gpu
def test_a_training_step_in_a_graph():
    """Captured once, replayed on other ids, groups and teachers, with eager work between the replays."""
    args = [t.to(DEV) for t in step_inputs(2)]
    args[3] = args[3].clone()
    WHOLE[args[0].shape[0]] = torch.tensor([0, args[0].shape[0]], device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*args)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(*args)
    for seed in (2, 3, 4, 3):
        for dst, src in zip(args, step_inputs(seed)):
            dst.copy_(src)
        eager = [t.clone() for t in step(*args)]
        torch.cuda.synchronize()
        for _ in range(2):
            for t in captured:
                t.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(captured, eager))


@gpu
def test_calls_on_another_stream():
    """Everything a call allocates by itself belongs to the stream it goes to."""
    args = step_inputs(5)
    ids, table, ptr, order, w1, b1, w2, top_ids, top, weight = (t.to(DEV) for t in args)
    want = step(ids, table, ptr, order, w1, b1, w2, top_ids, top, weight)
    x = binding.mgg_embed(ids[order], table, scale=2.0)
    hidden = binding.mgg_update_grouped(ptr, x, w1, b1, "relu")
    dz = torch.randn_like(hidden)
    logits = torch.randn(ids.shape[0], 47, device=DEV)
    torch.cuda.synchronize()
    wants = [x, hidden, *binding.mgg_update_grouped_grad(ptr, dz, x, w1, "relu", out=hidden, need_bias=True), binding.mgg_embed_grad(ids, x, 300),
             *binding.mgg_distill_loss(logits, top_ids, top, need_grad=True)]
    sorted_ids = ids[order]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = [binding.mgg_embed(sorted_ids, table, scale=2.0, stream=s), binding.mgg_update_grouped(ptr, x, w1, b1, "relu", stream=s),
           *binding.mgg_update_grouped_grad(ptr, dz, x, w1, "relu", out=hidden, need_bias=True, stream=s), binding.mgg_embed_grad(ids, x, 300, stream=s),
           *binding.mgg_distill_loss(logits, top_ids, top, need_grad=True, stream=s)]
    scribble = [torch.full_like(t, float("nan")) for t in got]           # what the current stream allocates now is not theirs
    s.synchronize()
    torch.cuda.synchronize()
    assert all(bool(torch.isnan(t).all()) for t in scribble)
    assert all(torch.equal(a, b) for a, b in zip(got, wants))
    assert len(want) == 5


# a launch has fewer than 2^32 threads; what would need more is refused before anything is launched
LARGE_WS = dict(bytes=2 ** 62)
TOO_LARGE = [
    (embed_call, dict(n=2 ** 31 - 1, dim=2, ld=2, ldo=2, tt=1, ot=1)),
    (embed_grad_call, dict(n=2 ** 30, dim=1, ld=1, ldo=1, gt=1, **LARGE_WS)),
    (grouped_call, dict(n=2 ** 31 - 1, g=1, k=1, m=1, lda=1, ldo=1)),
    (grouped_call, dict(n=2 ** 31 - 1, g=1)),
    (grouped_call, dict(n=2 ** 31 - 1, g=1, m=128, ldo=128, at=1, wt=1, ot=1)),
    (grouped_grad_call, dict(n=2 ** 31 - 1, g=1, act=1, out=P, ldo=8, db=P, **LARGE_WS)),
    (grouped_grad_call, dict(g=65535, k=2 ** 22, m=1, ldg=1, lda=2 ** 22, da=None, db=P, **LARGE_WS)),
    (distill_call, dict(n=2 ** 31 - 2, **LARGE_WS)),
    (distill_call, dict(n=2 ** 25, c=4096, ldz=4096, ldg=4096, **LARGE_WS)),
    (distill_call, dict(n=2 ** 25, c=4096, ldz=4096, grad=None, ldg=0, **LARGE_WS)),
]


@pytest.mark.parametrize("call,change", TOO_LARGE, ids=lambda v: str(v) if isinstance(v, dict) else None)
def test_more_threads_than_a_launch_has_are_refused(call, change):
    assert call(**change) == UNSUPPORTED
    assert len(binding.lib().mgg_last_error()) > 0


def _some_calls(seed):
    """One call of every operator on inputs of its own; returns a function that makes the calls and gives their outputs."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, rows, dim, groups, d_out, classes, k = 12000, 701, 264, 6, 136, 1001, 9
    ids = torch.randint(-1, rows, (n,), device="cuda", generator=g)
    ids[::3] = seed % rows                                   # a common one, whose sum reaches over many chunks
    rnd = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    table, w, bias, up = rnd(rows, dim).bfloat16(), rnd(groups, dim, d_out).bfloat16(), rnd(groups, d_out), rnd(n, d_out).bfloat16()
    ptr = torch.tensor([0, 5, 5, 3000, 9000, 11000, n], device="cuda")
    logits, top, top_ids = rnd(n, classes), rnd(n, k), torch.randint(-1, classes, (n, k), device="cuda", generator=g)

    def call(stream=None):
        a = binding.mgg_embed(ids, table, scale=1.5, stream=stream)
        out = binding.mgg_update_grouped(ptr, a, w, bias, "relu", stream=stream)
        grads = binding.mgg_update_grouped_grad(ptr, up, a, w, "relu", out=out, need_bias=True, stream=stream)
        back = binding.mgg_embed_grad(ids, grads[0], rows, scale=1.5, stream=stream)
        loss, grad = binding.mgg_distill_loss(logits, top_ids, top, temperature=2.0, need_grad=True, stream=stream)
        return (a, out, *grads, back, loss, grad)

    return call


@pytest.mark.gpu
def test_the_same_call_gives_the_same_bits():
    call = _some_calls(1)
    first = call()
    for _ in range(3):
        for x, y in zip(first, call()):
            assert torch.equal(x, y)


@pytest.mark.gpu
def test_two_streams_at_once():
    calls, streams = [_some_calls(s) for s in (2, 3)], [torch.cuda.Stream() for _ in range(2)]
    alone = [c() for c in calls]
    torch.cuda.synchronize()
    for _ in range(4):
        both = [c(stream=s) for _ in range(2) for c, s in zip(calls, streams)]
        torch.cuda.synchronize()
        for i, got in enumerate(both):
            for x, y in zip(alone[i % 2], got):
                assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("counts,d_in,d_out", [((3, 0, 40, 1), 20, 12), ((700, 9, 300), 130, 65), ((5, 6), 2, 3)])
def test_linear_gradients_against_differences(counts, d_in, d_out):
    """Products and lookups are linear in their weights, so a central difference of any step is exact but for rounding: an output of d terms is
    off by (d + 2) 2^-24 of the sum of their magnitudes, and so is a gradient of as many.  Inputs lie on a grid of 2^-6, so that the
    steps are exact."""
    g = torch.Generator(device="cuda").manual_seed(5)
    grid = lambda *shape: (torch.randn(*shape, device="cuda", generator=g).clamp(-3, 3) * 64).round() / 64
    n, groups = sum(counts), len(counts)
    ptr = torch.tensor([0, *np.cumsum(counts)], device="cuda")
    a, w, up = grid(n, d_in), grid(groups, d_in, d_out), grid(n, d_out)
    grad_a, grad_w = binding.mgg_update_grouped_grad(ptr, up, a, w)
    eps = 2.0 ** -24
    absolute = lambda x, y: binding.mgg_update_grouped(ptr, x.abs(), y.abs()).double() * 1.001       # (fp32 itself, hence the 1.001)
    for x, grad, terms, step in ((a, grad_a, d_out, grid(n, d_in)), (w, grad_w, max(counts), grid(groups, d_in, d_out))):
        plus, minus = ((x + step, w), (x - step, w)) if x is a else ((a, x + step), (a, x - step))
        difference = (binding.mgg_update_grouped(ptr, *plus).double() - binding.mgg_update_grouped(ptr, *minus).double()) * up.double() / 2
        off = (d_in + 2) * eps * ((absolute(*plus) + absolute(*minus)) * up.double().abs()).sum() / 2
        size_a, size_w = binding.mgg_update_grouped_grad(ptr, up.abs(), a.abs(), w.abs())
        off += (terms + 2) * eps * ((size_a if x is a else size_w).double() * step.double().abs()).sum() * 1.001
        # (sums in 64 bits round by 2^-53 a term, some 2^-33 of what the above allows for)
        assert abs(float((grad.double() * step.double()).sum() - difference.sum())) <= float(off)
    rows = 37
    ids = torch.randint(-1, rows, (n,), device="cuda", generator=g)
    table, step, up = grid(rows, d_in), grid(rows, d_in), grid(n, d_in)
    difference = (binding.mgg_embed(ids, table + step).double() - binding.mgg_embed(ids, table - step).double()) * up.double() / 2
    grad = binding.mgg_embed_grad(ids, up, rows).double()
    off = (n + 2) * eps * (binding.mgg_embed_grad(ids, up.abs(), rows).double() * step.double().abs()).sum() * 1.001
    assert abs(float((grad * step.double()).sum() - difference.sum())) <= float(off)


@gpu
def test_rows_as_long_as_32_bits_count():
    """2^31 - 1 columns: the last vectors' columns, and what a loop's step adds to them, lie past 32 bits.  Values stand at both ends and in the
    middle, zeros elsewhere; the elements around the matrices stay as they were."""
    dim, rows, guard = 2 ** 31 - 1, 3, 4096
    marks = torch.tensor([0, 1, 511, 2 ** 30, 2 ** 30 + 1, *range(dim - 20, dim)], device=DEV)

    def guarded(n):
        buf = torch.full((2 * guard + n * dim,), 9.0, dtype=BF16, device=DEV)
        return buf, buf[guard: guard + n * dim].view(n, dim)

    def untouched(buf):
        return bool((buf[:guard] == 9).all()) and bool((buf[-guard:] == 9).all())

    values = (torch.arange(marks.numel(), device=DEV) + 1).to(BF16)
    grad = torch.zeros(3, dim, dtype=BF16, device=DEV)
    for i in range(3):
        grad[i, marks] = values * (i + 1)
    buf, out = guarded(rows)
    ids = torch.tensor([0, 2, 0], device=DEV)
    binding.mgg_embed_grad(ids, grad, rows, out=out)
    assert untouched(buf)
    for v, factor in enumerate((4, 0, 2)):
        assert torch.equal(out[v, marks], (values.float() * factor).to(BF16))
        assert int((out[v] != 0).sum()) == (marks.numel() if factor else 0)
    del buf, out
    buf, out = guarded(2)
    binding.mgg_embed(torch.tensor([2, -1], device=DEV), grad, out=out)
    assert untouched(buf) and torch.equal(out[0], grad[2]) and not bool((out[1] != 0).any())


class _KernelNode(ctypes.Structure):            # hipKernelNodeParams
    _fields_ = [("block", ctypes.c_uint * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3),
                ("params", ctypes.c_void_p), ("shared", ctypes.c_uint)]


def launches(call):
    """(blocks along the first axis, threads of a block) of every kernel that the call launches, from a graph that it is captured into."""
    with open("/proc/self/maps") as f:
        path = next(line.split()[-1] for line in f if "libamdhip64" in line)        # the runtime that torch has loaded
    hip = ctypes.CDLL(path)
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        kept = call()
    raw, count = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    shapes = []
    for node in nodes:
        kind, p = ctypes.c_int(-1), _KernelNode()
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0 and kind.value == 0          # a kernel
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0
        shapes.append((p.grid[0], p.block[0]))
    del kept
    return shapes


@gpu
@pytest.mark.parametrize("n,tile", [(25, 128), (37, 128), (100, 128), (128, 128), (129, 128), (255, 128), (256, 128), (300, 256), (512, 256)])
def test_one_group_of_few_rows_and_many_columns(n, tile):
    """A head of 32,000 columns.  Pieces of one group are known: 25 to 256 rows are one piece of 256 or two of 128, and 125 large tiles leave
    more of the chip idle than 250 or 500 medium ones.  (Blocks of 512 threads take large tiles, those of 256 medium ones.)"""
    d_in, d_out = 72, 32000
    g = torch.Generator().manual_seed(n)
    a, w = torch.randn(n, d_in, generator=g).bfloat16(), (torch.randn(1, d_in, d_out, generator=g) * d_in ** -0.5).bfloat16()
    ptr = torch.tensor([0, n])
    args = (ptr.to(DEV), a.to(DEV), w.to(DEV))
    ref, mag = grouped_reference(ptr, a, w, None, "none")
    assert_within(binding.mgg_update_grouped(*args), ref, (d_in + 2) * U * mag + half_step(BF16) * ref.abs())
    out = torch.empty(n, d_out, dtype=BF16, device=DEV)
    assert launches(lambda: binding.mgg_update_grouped(*args, out=out)) == [((n // tile + 1) * (d_out // tile), 2 * tile)]


def test_workspace_has_no_partial_sums_of_groups_that_are_one_piece():
    """A matrix per piece only for groups longer than a piece: at most 2 floor(n / step) of them, 256 rows to a piece at least."""
    grouped = binding.mgg_update_grouped_grad_workspace_bytes
    bias = lambda n, groups, d_out: (n // 64 + min(n, groups)) * d_out * 4          # of the columns' sums, 64 rows to a piece at least
    assert grouped(64, 64, 512, 1024, F32) <= bias(64, 64, 1024) + 1024
    assert grouped(255, 5, 602, 47, F32) <= bias(255, 5, 47) + 1024
    assert grouped(65536, 128, 1001, 1801, BF16) <= 8 * 1001 * 1801 * 4 + bias(65536, 128, 1801) + 1024           # (13,120 rows to a piece)
    assert grouped(1000, 1, 64, 64, BF16) >= 4 * 64 * 64 * 4


@gpu
@pytest.mark.parametrize("dtype,d_in,d_out", [(BF16, 64, 64), (F32, 40, 72), (BF16, 3, 20), (BF16, 130, 47)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_gradients_of_groups_of_one_piece_and_of_several(dtype, d_in, d_out, accumulate):
    """150 groups of lengths about multiples of a piece (256 rows here), in a workspace of just the size that is asked for."""
    rng = np.random.default_rng(d_in)
    counts = rng.choice([0, 1, 255, 256, 257, 300, 512, 513, 1100], 150).tolist()
    n, groups = sum(counts), len(counts)
    g = torch.Generator().manual_seed(d_out)
    a, dz, w = torch.randn(n, d_in, generator=g).to(dtype), torch.randn(n, d_out, generator=g).to(dtype), torch.zeros(groups, d_in, d_out, dtype=dtype)
    into, into_b = torch.randn(groups, d_in, d_out, generator=g), torch.randn(groups, d_out, generator=g)
    ptr = group_ptr(counts)
    (_, dw, db), (_, mw, mb) = grouped_grad_reference(ptr, dz, a, w)
    if accumulate:
        dw, db, mw, mb = dw + into, db + into_b, mw + into.abs(), mb + into_b.abs()
    need = binding.mgg_update_grouped_grad_workspace_bytes(n, groups, d_in, d_out, dtype)
    buf = torch.full((need + 8192,), 0xff, dtype=torch.uint8, device=DEV)           # (NaN wherever it is read before it is written)
    args = [t.to(DEV) for t in (ptr, dz, a, w)]
    for _ in range(2):
        _, gw, gb = binding.mgg_update_grouped_grad(*args, need_a=False, need_bias=True, grad_w=into.to(DEV), grad_bias=into_b.to(DEV), accumulate=accumulate,
                                                    workspace=buf[4096: 4096 + need])
        assert bool((buf[:4096] == 0xff).all()) and bool((buf[4096 + need:] == 0xff).all())
        terms = (max(counts) + 3) * U
        assert_within(gw, dw, terms * mw + half_step(F32) * dw.abs(), "grad_w")
        assert_within(gb, db, terms * mb + half_step(F32) * db.abs(), "grad_bias")


def test_accumulating_into_nothing_is_refused():
    ptr, a, w = torch.zeros(3, dtype=torch.int64), torch.zeros(4, 8), torch.zeros(2, 8, 8)
    with pytest.raises(ValueError, match="accumulate"):
        binding.mgg_update_grouped_grad(ptr, a, a, w, need_bias=True, accumulate=True)
    for given in (dict(grad_w=torch.zeros(2, 8, 8)), dict(grad_bias=torch.zeros(2, 8))):         # (these go on to the refusal of host tensors)
        with pytest.raises(TypeError):
            binding.mgg_update_grouped_grad(ptr, a, a, w, need_bias=True, accumulate=True, **given)


# ---- kernels at lengths where their loops come round ----------------------------------------------------------
STEPS = [64, 72, 128, 136, 192, 200, 256, 320, 328, 512, 1000]      # a step of the sum is 64 long


@gpu
@pytest.mark.parametrize("depth", STEPS)
def test_large_tiles_over_one_to_many_steps(depth):
    """256 x 256 tiles of the forward product and of the rows' gradient (a block has 512 threads there): sums of one step, of two to
    sixteen, whole and with a remainder, over groups that end in and at tiles."""
    counts, wide = [1500, 0, 700, 1, 255, 256, 257, 1031], 2056
    n, groups = sum(counts), len(counts)
    g = torch.Generator().manual_seed(depth)
    a, w = torch.randn(n, depth, generator=g).bfloat16(), (torch.randn(groups, depth, wide, generator=g) * depth ** -0.5).bfloat16()
    ptr, bias = group_ptr(counts), torch.randn(groups, wide, generator=g)
    grid = [((n // 256 + groups) * 9, 512)]
    ref, mag = grouped_reference(ptr, a, w, bias, "none")
    args = (ptr.to(DEV), a.to(DEV), w.to(DEV), bias.to(DEV))
    out = torch.empty(n, wide, dtype=F32, device=DEV)
    assert_within(binding.mgg_update_grouped(*args, out=out), ref, (depth + 2) * U * mag + half_step(F32) * ref.abs(), "out")
    assert launches(lambda: binding.mgg_update_grouped(*args, out=out)) == grid
    # the same product as a rows' gradient: dz = a, the weights turned
    turned, rows = w.transpose(1, 2).contiguous().to(DEV), torch.zeros(n, wide, dtype=BF16, device=DEV)
    call = dict(need_w=False, grad_a=out, workspace=torch.empty(binding.mgg_update_grouped_grad_workspace_bytes(n, groups, wide, depth, BF16), dtype=torch.uint8, device=DEV))
    ref, mag = grouped_reference(ptr, a, w, None, "none")
    got, _ = binding.mgg_update_grouped_grad(args[0], args[1], rows, turned, **call)
    assert_within(got, ref, (depth + 2) * U * mag + half_step(F32) * ref.abs(), "grad_a")
    assert launches(lambda: binding.mgg_update_grouped_grad(args[0], args[1], rows, turned, **call)) == grid


@gpu
@pytest.mark.parametrize("tw,accumulate", [(F32, False), (F32, True), (BF16, False)])
def test_large_tiles_of_weight_gradients_over_none_to_many_steps(tw, accumulate):
    """Groups of 0 to 1000 rows, a step being 64 of them: exactly one to seven steps, and with a remainder."""
    counts, d_in, d_out = [1000, 192, 128, 256, 64, 320, 0, 1, 63, 65, 129, 7, 0, 200, 384, 449, 72, 500, 130, 191], 1024, 1032
    n, groups = sum(counts), len(counts)
    g = torch.Generator().manual_seed(7)
    a, dz = torch.randn(n, d_in, generator=g).bfloat16(), torch.randn(n, d_out, generator=g).bfloat16()
    into = torch.randn(groups, d_in, d_out, generator=g).to(tw)
    ptr, w = group_ptr(counts), torch.zeros(groups, d_in, d_out, dtype=BF16)
    (_, ref, _), (_, mag, _) = grouped_grad_reference(ptr, dz, a, w)
    if accumulate:
        ref, mag = ref + into, mag + into.abs()
    args = [t.to(DEV) for t in (ptr, dz, a, w)]
    call = dict(need_a=False, grad_w=into.to(DEV), accumulate=accumulate,
                workspace=torch.empty(binding.mgg_update_grouped_grad_workspace_bytes(n, groups, d_in, d_out, BF16), dtype=torch.uint8, device=DEV))
    got = binding.mgg_update_grouped_grad(*args, **call)[1]
    assert_within(got, ref, (torch.tensor(counts)[:, None, None] + 3) * U * mag + half_step(tw) * ref.abs(), "grad_w")
    assert launches(lambda: binding.mgg_update_grouped_grad(*args, **call)) == [(groups * 4 * 5, 512)]


@gpu
@pytest.mark.parametrize("d_in,d_out", [(256, 1024), (250, 1001), (1000, 1500)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_row_or_two_to_each_of_many_groups(d_in, d_out, dtype):
    """Four wavefronts share the sum of a tile of 32 rows where there are 512 tiles and more: a serving step over 64 groups, 23 of them idle."""
    rng = np.random.default_rng(d_in)
    counts = np.bincount(rng.permutation(64)[rng.integers(0, 41, 64)], minlength=64).tolist()
    n, groups = sum(counts), len(counts)
    g = torch.Generator().manual_seed(d_out)
    a, dz = torch.randn(n, d_in, generator=g).to(dtype), torch.randn(n, d_out, generator=g).to(dtype)
    w, ptr = (torch.randn(groups, d_in, d_out, generator=g) * d_in ** -0.5).to(dtype), group_ptr(counts)
    args = [t.to(DEV) for t in (ptr, dz, a, w)]
    ref, mag = grouped_reference(ptr, a, w, None, "none")
    out = torch.empty(n, d_out, dtype=dtype, device=DEV)
    assert_within(binding.mgg_update_grouped(args[0], args[2], args[3], out=out), ref, (d_in + 2) * U * mag + half_step(dtype) * ref.abs(), "out")
    assert launches(lambda: binding.mgg_update_grouped(args[0], args[2], args[3], out=out)) == [((n // 32 + 64) * -(-d_out // 64), 256)]
    refs, mags = grouped_grad_reference(ptr, dz, a, w)
    for name, x, r, m, k in zip(("grad_a", "grad_w"), binding.mgg_update_grouped_grad(*args), refs, mags, (d_out, max(counts))):
        assert_within(x, r, (k + 3) * U * m + half_step(x.dtype) * r.abs(), name)


@gpu
@pytest.mark.parametrize("n,classes,k,dtype,shape", [(64, 40001, 7, F32, (64, 1024)), (66, 65536, 3, F32, (66, 1024)), (64, 131072, 5, BF16, (64, 1024)),
                                                     (65, 65544, 9, BF16, (65, 1024)), (3, 16384, 4, F32, (3, 1024)), (3, 8192, 4, F32, (3, 256)), (4, 8193, 4, F32, (4, 1024)),
                                                     (5, 1025, 3, F32, (5, 256)), (5, 2049, 3, BF16, (5, 256))])
def test_distill_rows_at_the_ends_of_what_registers_hold(n, classes, k, dtype, shape):
    z, ids, top, weight = draw_distill(n, classes, k, classes, dtype, F32)
    loss, grad, loss_bound, grad_bound = distill_reference(z, ids, top, 2.0, weight)
    args = [t.to(DEV) for t in (z, ids, top)]
    call = dict(temperature=2.0, row_weight=weight.to(DEV), loss=torch.empty(n, device=DEV), grad=torch.empty(n, classes, dtype=dtype, device=DEV),
                workspace=torch.empty(binding.mgg_distill_workspace_bytes(n, classes), dtype=torch.uint8, device=DEV))
    got, got_grad = binding.mgg_distill_loss(*args, **call)
    assert_within(got, loss, loss_bound + half_step(F32) * loss.abs(), "loss")
    assert_within(got_grad, grad, grad_bound + half_step(dtype) * grad.abs() + 1e-37, "gradient")
    assert launches(lambda: binding.mgg_distill_loss(*args, **call)) == [shape]


@gpu
def test_a_training_step_around_the_aggregation():
    """Lookup, GCN aggregation, Update by node type, class head, loss, and back.  On a graph whose edges go both ways the normalised adjacency is
    symmetric, so the aggregation's gradient is the aggregation of the gradient.  Against autograd in float64; fp32 throughout: seven
    products and sums of at most 700 terms one after the other, 2-norms within 7 * 700 * 2^-23."""
    ids, table, _, _, w1, b1, w2, top_ids, top, weight = step_inputs(6)
    n, t = ids.shape[0], 2.0
    rng = np.random.default_rng(6)
    adjacency = np.triu(rng.random((n, n)) < 0.02, 1)
    adjacency = adjacency | adjacency.T
    row_ptr, col = np.concatenate([[0], adjacency.sum(1).cumsum()]), np.nonzero(adjacency)[1]
    looped = torch.from_numpy(adjacency + np.eye(n))
    scale = looped.sum(1).rsqrt()
    a_hat = looped * scale[:, None] * scale[None, :]
    ptr = torch.tensor([0, 120, 120, 400, 650, n])                       # nodes stand type by type
    leaves = [x.double().requires_grad_() for x in (table, w1, b1, w2)]
    h = a_hat @ leaves[0][ids]
    hidden = torch.cat([torch.relu(h[int(ptr[g]):int(ptr[g + 1])] @ leaves[1][g] + leaves[2][g]) for g in range(w1.shape[0])])
    log_q, log_p = torch.log_softmax(hidden @ leaves[3] / t, 1), torch.log_softmax(top.double() / t, 1)
    want = weight.double() * t * t * (log_p.exp() * (log_p - log_q.gather(1, top_ids))).sum(1)
    want.sum().backward()

    part = binding.mgg_build_partition(row_ptr, col)
    ids, table, w1, b1, w2, top_ids, top, weight, ptr = (x.to(DEV) for x in (ids, table, w1, b1, w2, top_ids, top, weight, ptr))
    h = binding.mgg_aggregate(part, "gcn", binding.mgg_embed(ids, table))
    hidden = binding.mgg_update_grouped(ptr, h, w1, b1, "relu")
    loss, dlogits = binding.mgg_distill_loss(binding.mgg_update(hidden, w2), top_ids, top, temperature=t, row_weight=weight, need_grad=True)
    dhidden, dw2 = binding.mgg_update_grouped_grad(torch.tensor([0, n], device=DEV), dlogits, hidden, w2[None])
    dh, dw1, db1 = binding.mgg_update_grouped_grad(ptr, dhidden, h, w1, "relu", out=hidden, need_bias=True)
    dtable = binding.mgg_embed_grad(ids, binding.mgg_aggregate(part, "gcn", dh), table.shape[0])
    for name, x, ref in zip(("loss", "table", "w1", "b1", "w2"), (loss, dtable, dw1, db1, dw2[0]), [want.detach()] + [leaf.grad for leaf in leaves]):
        rel = float((x.double().cpu() - ref).norm() / ref.norm())
        assert rel < 7 * 700 * U, (name, rel)


@gpu
@pytest.mark.parametrize("offsets", [[0, 2000, 500, 2000], [0, 2000] * 40, [0, 2000, 1999, 3, 1500, 0, 5000, -7, 700]])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_overlapping_groups_of_several_pieces_stay_inside_the_workspace(offsets, dtype):
    """Such groups have more pieces than ascending offsets could have; what they compute is not defined, where it is written is."""
    n, d, groups = 2000, 24, len(offsets) - 1
    ptr = torch.tensor(offsets, device=DEV)
    one = lambda *shape: torch.ones(*shape, dtype=dtype, device=DEV)
    need = binding.mgg_update_grouped_grad_workspace_bytes(n, groups, d, d, dtype, act="relu")
    space, around = torch.full((need + 8192,), 0x3c, dtype=torch.uint8, device=DEV), torch.full((3 * n, d), 5.0, dtype=dtype, device=DEV)
    around_w = torch.full((3 * groups, d, d), 5.0, device=DEV)
    binding.mgg_update_grouped_grad(ptr, one(n, d), one(n, d), one(groups, d, d), "relu", out=one(n, d), need_bias=True, grad_a=around[n:2 * n],
                                    grad_w=around_w[groups:2 * groups], workspace=space[4096: 4096 + need])
    torch.cuda.synchronize()
    assert bool((space[:4096] == 0x3c).all()) and bool((space[4096 + need:] == 0x3c).all())
    assert bool((around[:n] == 5).all()) and bool((around[2 * n:] == 5).all())
    assert bool((around_w[:groups] == 5).all()) and bool((around_w[2 * groups:] == 5).all())
