"""The operators around the expert layer against plain implementations in 64 bits.

Where the tolerances come from.  u is half a unit in the last place of the output's type (bf16 2^-8, f16 2^-11 and
2^-25 absolute below its normal range, f32 2^-24).  A kernel sums a row in 32 bits, at most 64 values in sequence per thread and then
a tree of ten levels: relative error at most 80 * 2^-24 = 4.8e-6 of the sum of magnitudes.  rstd is a square root of such
a sum (half of that); everything after it is a handful of products of 2^-24 each.  So values before the last rounding
are within 6e-6 of their magnitudes' sum, and 1e-5 is used where two such sums meet.  A value in 8 bits is off by
half a step, and by 127 times the relative error of value and scale: (0.5 + 127 * 1.2e-5) steps < 0.502.
"""
import ctypes
import math

import pytest

from paper_2607_19539_b200 import binding as B

torch = pytest.importorskip("torch")
from paper_2607_19539_b200 import ops  # noqa: E402

gpu = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {t: torch.finfo(t).eps / 2 for t in (BF16, F16, F32)}
FLOOR = {BF16: 1e-38, F16: 2.0 ** -25, F32: 1e-38}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def guarded(rows, cols, dtype, pad=0, shift=0, fill=None):
    """A [rows, cols] view whose rows lie `pad` apart and start `shift` elements in, and the buffer around it."""
    full = torch.full((rows + 2, cols + pad + shift), 77 if dtype is torch.int8 else 7.5, dtype=dtype, device="cuda")
    return full[1:rows + 1, shift:shift + cols], full


def untouched(full, view):
    keep = full.clone()
    rows, cols = view.shape
    shift = view.storage_offset() % full.stride(0)
    keep[1:rows + 1, shift:shift + cols] = full.reshape(-1)[0]
    return bool((keep == full.reshape(-1)[0]).all())


def close(got, want, bound):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), (int(bad.sum()), got[bad][:4].tolist(), want[bad][:4].tolist(), float(((got - want).abs() / bound)[bad].max()))


# ------------------------------------------------------------------------------------------------ norm

def norm64(h, w, eps):
    h, w = h.double(), w.double()
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * w, rstd


WIDTHS = [1, 7, 8, 33, 64, 127, 256, 1000, 1408, 4096, 4099, 8192, 10248, 16384, 32768]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", WIDTHS)
def test_add_norm(d, dtype):
    for case, (rows, pad, shift) in enumerate([(1, 0, 0), (3, 8, 0), (5, 3, 1), (301, 0, 0)]):
        g = gen(d * 10 + case)
        x, fx = guarded(rows, d, dtype, pad, shift)
        r, fr = guarded(rows, d, dtype, pad, shift)
        x.copy_(normal(g, (rows, d), dtype))
        r.copy_(normal(g, (rows, d), dtype, 2.0))
        w = normal(g, (d,), F32 if case % 2 else dtype) + 1
        h_out, fh = guarded(rows, d, dtype, pad, shift)
        y, fy = guarded(rows, d, dtype, pad, shift)
        q, fq = guarded(rows, d, torch.int8, pad, shift)
        scale, rstd = torch.full((rows,), -1.0, device="cuda"), torch.full((rows,), -1.0, device="cuda")
        ops.moe_ovl_add_norm(x=x, residual=r, weight=w, eps=1e-5, residual_out=h_out, y=y, q=q, scale=scale, rstd=rstd)
        h = (x.float() + r.float()).to(dtype)
        assert torch.equal(h_out, h)
        v, rs = norm64(h, w, 1e-5)
        close(rstd, rs, 4e-6 * rs)
        close(y, v, (U[dtype] + 6e-6) * v.abs() + FLOOR[dtype])
        want = v.abs().amax(1) / 127
        close(scale, want, 6e-6 * want)
        close(q.double() * scale.double()[:, None], v, 0.502 * want[:, None])
        assert bool((q.abs().amax(1) == 127).all())
        for full, view in ((fh, h_out), (fy, y), (fq, q)):
            assert untouched(full, view)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_add_norm_without_residual_and_single_outputs(dtype):
    g = gen(3)
    x, w = normal(g, (37, 520), dtype), normal(g, (520,), dtype)
    v, rs = norm64(x, w, 1e-6)
    y = torch.empty_like(x)
    ops.moe_ovl_add_norm(x=x, weight=w, y=y)
    close(y, v, (U[dtype] + 6e-6) * v.abs() + FLOOR[dtype])
    rstd = torch.empty(37, device="cuda")
    ops.moe_ovl_add_norm(x=x, weight=w, rstd=rstd)
    close(rstd, rs, 4e-6 * rs)
    h = torch.empty_like(x)                                 # the sum alone, and in place
    ops.moe_ovl_add_norm(x=x, residual=y, weight=w, residual_out=h)
    z = y.clone()
    ops.moe_ovl_add_norm(x=x, residual=z, weight=w, residual_out=z)
    assert torch.equal(h, z) and torch.equal(h, (x.float() + y.float()).to(dtype))
    z = x.clone()
    ops.moe_ovl_add_norm(x=z, weight=w, y=z)
    assert torch.equal(z, y)
    ops.moe_ovl_add_norm(x=x[:0], weight=w, y=y[:0])        # no rows


@gpu
@pytest.mark.parametrize("d", [40, 4096, 4097])
def test_add_norm_rows_out_of_the_ordinary(d):
    """Zeros, one large value, values below the range of the scale, NaN and infinity: each row by itself."""
    g = gen(d)
    x = normal(g, (8, d), F32)
    x[0] = 0
    x[1] = 0
    x[1, d // 2] = 1e15
    x[2] *= 1e-36
    x[3, 3] = float("nan")
    x[4, 5] = float("inf")
    x[5] = 1e25                                             # the square is beyond the type: 1 / inf = 0
    w = torch.ones(d, device="cuda")
    y, q = torch.empty_like(x), torch.full((8, d), 9, dtype=torch.int8, device="cuda")
    scale = torch.empty(8, device="cuda")
    ops.moe_ovl_add_norm(x=x, weight=w, eps=1e-6, y=y, q=q, scale=scale)
    assert not y[0].any() and not q[0].any() and scale[0] == 0
    assert q[1, d // 2] == 127 and q[1].abs().sum() == 127
    close(scale[1:2], torch.tensor([math.sqrt(d) / 127], device="cuda"), 1e-4)
    assert scale[2] == 0 and not q[2].any()                 # |v| < 1e-32
    assert bool(y[3].isnan().all()) and bool(scale[3].isnan()) and not q[3].any()
    assert bool(y[4, 5].isnan()) and not y[4, 6:].any() and bool(scale[4].isnan()) and not q[4].any()
    assert not y[5].any() and scale[5] == 0
    v, _ = norm64(x[6:], w, 1e-6)
    close(y[6:], v, 6e-6 * v.abs())
    wn = w.clone()
    wn[1] = float("nan")
    ops.moe_ovl_add_norm(x=x[6:], weight=wn, q=q[6:], scale=scale[6:])
    assert bool(scale[6:].isnan().all()) and not q[6:].any()


def norm_backward64(dy, h, w, rstd, dr):
    dy, h, w, rstd = dy.double(), h.double(), w.double(), rstd.double()[:, None]
    n, gg = h * rstd, dy * w
    dx = rstd * (gg - n * (gg * n).mean(1, keepdim=True))
    size = rstd * (gg.abs() + n.abs() * (gg * n).abs().mean(1, keepdim=True))
    if dr is not None:
        dx, size = dx + dr.double(), size + dr.double().abs()
    return dx, (dy * n).sum(0), size, (dy * n).abs().sum(0)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", WIDTHS)
def test_add_norm_backward(d, dtype):
    for case, (rows, pad, shift) in enumerate([(1, 0, 0), (3, 8, 0), (6, 3, 1), (149, 0, 0), (1303, 0, 0)]):
        if rows * d > 20e6:
            continue
        g = gen(d * 10 + case)
        make = lambda: guarded(rows, d, dtype, pad, shift)  # noqa: E731
        (dy, _), (h, _), (dr, _), (dx, full) = make(), make(), make(), make()
        dy.copy_(normal(g, (rows, d), dtype))
        h.copy_(normal(g, (rows, d), dtype, 1.5))
        dr.copy_(normal(g, (rows, d), dtype))
        w = normal(g, (d,), F32 if case % 2 else dtype) + 1
        rstd = (1.0 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
        dw = torch.full((d,), 5.0, device="cuda")
        ws = torch.full((ops.moe_ovl_add_norm_workspace_bytes(rows, d) // 4 + 64,), 3.0, device="cuda")
        use = dr if case != 1 else None
        ops.moe_ovl_add_norm_backward(dy=dy, h=h, weight=w, rstd=rstd, d_residual=use, dx=dx, dweight=dw, workspace=ws[:-64])
        want, dw_want, size, dw_size = norm_backward64(dy, h, w, rstd, use)
        close(dx, want, U[dtype] * want.abs() + 1e-5 * size + FLOOR[dtype])
        close(dw, dw_want, 1e-5 * dw_size + 1e-30)
        assert bool((ws[-64:] == 3).all()) and untouched(full, dx)
        dw2, (dx2, _) = torch.empty_like(dw), make()
        ops.moe_ovl_add_norm_backward(dy=dy, h=h, weight=w, rstd=rstd, d_residual=use, dx=dx2, dweight=dw2, workspace=ws)
        assert torch.equal(dw, dw2) and torch.equal(dx, dx2)        # the same bits
        ops.moe_ovl_add_norm_backward(dy=dy, h=h, weight=w, rstd=rstd, d_residual=use, dx=dy)     # in place, without dweight
        assert torch.equal(dy, dx)


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("d", [3, 9, 33, 127, 250, 255, 513, 1001, 2047, 4097, 8190])
def test_add_norm_and_gradient_of_ragged_rows(d, dtype):
    """Rows whose length or distance is no multiple of 16 bytes, from aligned bases, more of them than blocks; then with matrices that do
    not agree on where a row begins."""
    g = gen(d)
    for rows, pads in ((2, (0, 0, 0)), (1900, (0, 0, 0)), (2500, (8, 16, 0)), (700, (1, 2, 5))):
        wide = lambda pad, t=dtype: torch.full((rows, d + pad), 7, dtype=t, device="cuda")  # noqa: E731
        x, r, h, y = wide(pads[0]), wide(pads[1]), wide(pads[2]), wide(pads[0])
        q, scale, rstd = wide(pads[1], torch.int8), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        cut = lambda m: m[:, :d]  # noqa: E731
        cut(x).copy_(normal(g, (rows, d), dtype))
        cut(r).copy_(normal(g, (rows, d), dtype))
        w = normal(g, (d,), dtype) + 1
        ops.moe_ovl_add_norm(x=cut(x), residual=cut(r), weight=w, residual_out=cut(h), y=cut(y), q=cut(q), scale=scale, rstd=rstd)
        assert torch.equal(cut(h), (cut(x).float() + cut(r).float()).to(dtype))
        v, rs = norm64(cut(h), w, 1e-6)
        close(rstd, rs, 4e-6 * rs)
        close(cut(y), v, (U[dtype] + 6e-6) * v.abs() + FLOOR[dtype])
        close(cut(q).double() * scale.double()[:, None], v, 0.502 * v.abs().amax(1, keepdim=True) / 127)
        dy, dx, dw = wide(pads[1]), wide(pads[0]), torch.empty(d, device="cuda")
        cut(dy).copy_(normal(g, (rows, d), dtype))
        ws = torch.empty(ops.moe_ovl_add_norm_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
        ops.moe_ovl_add_norm_backward(dy=cut(dy), h=cut(h), weight=w, rstd=rstd, d_residual=cut(r), dx=cut(dx), dweight=dw, workspace=ws)
        want, dw_want, size, dw_size = norm_backward64(cut(dy), cut(h), w, rstd, cut(r))
        close(cut(dx), want, U[dtype] * want.abs() + 1e-5 * size + FLOOR[dtype])
        close(dw, dw_want, 1e-5 * dw_size + 1e-30)
        for m, pad in ((h, pads[2]), (y, pads[0]), (q, pads[1]), (dx, pads[0])):
            assert pad == 0 or bool((m[:, d:] == 7).all())


@gpu
def test_add_norm_backward_against_differences():
    """The kernel's gradient along random directions against central differences of the 64-bit forward pass."""
    rows, d, eps = 5, 333, 1e-3
    g = gen(1)
    x, r, w = normal(g, (rows, d), F32), normal(g, (rows, d), F32), normal(g, (d,), F32) + 1
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    ops.moe_ovl_add_norm(x=x, residual=r, weight=w, eps=eps, residual_out=h, y=y, rstd=rstd)
    dy, dh = normal(g, (rows, d), F32), normal(g, (rows, d), F32)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(ops.moe_ovl_add_norm_workspace_bytes(rows, d), dtype=torch.uint8, device="cuda")
    ops.moe_ovl_add_norm_backward(dy=dy, h=h, weight=w, rstd=rstd, d_residual=dh, dx=dx, dweight=dw, workspace=ws)

    def loss(hh, ww):
        return float((norm64(hh, ww, eps)[0] * dy.double()).sum() + (hh * dh.double()).sum())

    for _ in range(4):
        a = torch.randn((rows, d), generator=g, device="cuda", dtype=torch.float64)
        b = torch.randn(d, generator=g, device="cuda", dtype=torch.float64)
        t = 1e-5
        num = (loss(h.double() + t * a, w.double() + t * b) - loss(h.double() - t * a, w.double() - t * b)) / (2 * t)
        got = float((dx.double() * a).sum() + (dw.double() * b).sum())
        # 32-bit gradients summed over ~1700 entries of size ~1 with random signs; differences are good to t^2
        assert abs(num - got) <= 1e-5 * float((dx.double() * a).abs().sum() + (dw.double() * b).abs().sum())


@gpu
def test_add_norm_backward_no_rows():
    dw = torch.full((64,), 3.0, device="cuda")
    e = torch.empty((0, 64), device="cuda")
    ops.moe_ovl_add_norm_backward(dy=e, h=e, weight=torch.ones(64, device="cuda"), rstd=torch.empty(0, device="cuda"), dx=e, dweight=dw)
    assert not dw.any()


# ------------------------------------------------------------------------------------------------ gated activation

@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("f", WIDTHS)
def test_swiglu_quant(f, dtype):
    for case, (rows, pad, shift) in enumerate([(1, 0, 0), (4, 8, 0), (5, 3, 1), (299, 0, 0)]):
        g = gen(f * 10 + case)
        x, _ = guarded(rows, 2 * f, dtype, pad, shift)
        x.copy_(normal(g, (rows, 2 * f), dtype, 3.0))
        q, full = guarded(rows, f, torch.int8, pad, shift)
        scale = torch.empty(rows, device="cuda")
        ops.moe_ovl_swiglu_quant(gate_up=x, q=q, scale=scale)
        a, b = x[:, :f].double(), x[:, f:].double()
        v = a * torch.sigmoid(a) * b
        want = v.abs().amax(1) / 127
        close(scale, want, 6e-6 * want)
        close(q.double() * scale.double()[:, None], v, 0.502 * want[:, None])
        assert untouched(full, q)


@gpu
def test_swiglu_quant_rows_out_of_the_ordinary():
    x = torch.ones((6, 2 * 24), device="cuda")
    x[0] = 0
    x[1, 0] = float("nan")
    x[2, 24 + 3] = float("inf")
    x[3, :24] = -200.0                                      # exp overflows: silu is -0
    x[4, :24] = 200.0
    x[4, 24:] = torch.arange(24, device="cuda")
    x[5, :24] = float("-inf")                               # -inf * 0 is not a number
    q, scale = torch.full((6, 24), 9, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    ops.moe_ovl_swiglu_quant(gate_up=x, q=q, scale=scale)
    assert scale[0] == 0 and not q[0].any()
    assert bool(scale[1].isnan()) and not q[1].any()
    assert bool(scale[2].isinf()) and not q[2].any()
    assert scale[3] == 0 and not q[3].any()
    close(scale[4:5], torch.tensor([200.0 * 23 / 127], device="cuda"), 1e-3)
    assert q[4, 23] == 127 and q[4, 0] == 0
    assert bool(scale[5].isnan()) and not q[5].any()
    ops.moe_ovl_swiglu_quant(gate_up=x[:0], q=q[:0], scale=scale[:0])


# ------------------------------------------------------------------------------------------------ router

def route64(logits, k, score, bias, groups, top_groups, group_best, renorm, c):
    """Row by row from the definition; also each row's smallest gap between two different choices (ties are exact)."""
    lg = logits.double().cpu()
    lg = torch.where(lg.isnan(), torch.tensor(-math.inf, dtype=torch.float64), lg)
    big = 3.4028234663852886e38
    lg = torch.minimum(lg, torch.tensor(big, dtype=torch.float64))
    t, e = lg.shape
    idx, gate = torch.full((t, k), -1, dtype=torch.int32), torch.zeros((t, k), dtype=torch.float64)
    gaps = []
    for i in range(t):
        gap = math.inf
        row = lg[i]
        live = row > -math.inf
        if score == "sigmoid":
            s = torch.sigmoid(row)
        elif live.any():
            z = torch.exp(row - row.max())
            s = z / z.sum()
        else:
            s = torch.zeros(e, dtype=torch.float64)
        by_score = bias is not None or (groups > 1 and group_best == 2)
        ch = s.clone() if by_score else row.clone()
        if bias is not None:
            bb = bias.double().cpu()
            ch = ch + torch.where(bb.isnan(), torch.tensor(-math.inf, dtype=torch.float64), bb)
        ch[~live] = -math.inf
        values = sorted(set(ch[ch > -math.inf].tolist()))
        gap = min([gap] + [b - a for a, b in zip(values, values[1:])])
        if groups > 1:
            gv = []
            for j in range(groups):
                m = sorted([v for v in ch[j * e // groups:(j + 1) * e // groups].tolist() if v > -math.inf], reverse=True)[:group_best]
                gv.append(sum(m) if m else -math.inf)
            values = sorted(set(v for v in gv if v > -math.inf))
            gap = min([gap] + [b - a for a, b in zip(values, values[1:])])
            kept = sorted(range(groups), key=lambda j: (-gv[j], j))[:top_groups]
            for j in range(groups):
                if j not in kept:
                    ch[j * e // groups:(j + 1) * e // groups] = -math.inf
        gaps.append(gap)
        order = sorted([j for j in range(e) if ch[j] > -math.inf], key=lambda j: (-float(ch[j]), j))[:k]
        if not order:
            continue
        if renorm and score == "softmax":
            z = torch.exp(row[order] - row[order].max())
            gt = z / z.sum()
        else:
            gt = s[order]
            if renorm:
                gt = gt / gt.sum() if gt.sum() > 0 else torch.zeros_like(gt)
        idx[i, :len(order)] = torch.tensor(order, dtype=torch.int32)
        gate[i, :len(order)] = c * gt
    return idx, gate, torch.tensor(gaps)


def call_route(logits, k, score="softmax", bias=None, groups=1, top_groups=1, group_best=1, renorm=True, c=1.0, counts=True):
    t, e = logits.shape
    expert = torch.full((t, k), -9, dtype=torch.int32, device="cuda")
    gate = torch.full((t, k), -9.0, device="cuda")
    n = torch.full((e,), -9, dtype=torch.int32, device="cuda") if counts else None
    ops.moe_ovl_route(logits=logits, expert=expert, gate=gate, counts=n, bias=bias, score=ops.SCORES[score], num_groups=groups,
                      top_groups=top_groups, group_best=group_best, renormalise=renorm, gate_scale=c)
    return expert, gate, n


def check_route(logits, k, **kw):
    bias = kw.get("bias")
    idx, gate, gap = route64(logits, k, kw.get("score", "softmax"), bias, kw.get("groups", 1), kw.get("top_groups", 1), kw.get("group_best", 1),
                             kw.get("renorm", True), kw.get("c", 1.0))
    clear = gap > 1e-6              # the other rows hold a near-tie that 32 bits need not tell apart
    assert int(clear.sum()) * 2 >= len(clear)
    got_i, got_g, got_n = (v.cpu() for v in call_route(logits, k, **kw))
    assert torch.equal(got_i[clear], idx[clear])
    # exp and the sums over up to 1024 scores: 1e-5 covers 2 ulp of exp and 40 roundings of the sum
    close(got_g[clear], gate[clear], 1e-5 * gate[clear].abs() + 1e-37)
    assert torch.equal(got_n.long(), torch.bincount(got_i[got_i >= 0].flatten().long(), minlength=logits.shape[1]))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("e,k", [(1, 1), (2, 2), (8, 2), (17, 5), (32, 32), (60, 4), (64, 6), (100, 9), (128, 8), (160, 6), (256, 8), (384, 8), (500, 10),
                                 (512, 32), (1024, 8)])
def test_route_softmax(e, k, dtype):
    g = gen(e)
    for rows in (1, 9, 70):
        # a coarse grid: equal logits are frequent, different ones differ clearly
        logits = torch.randint(-40, 41, (rows, e), generator=g, device="cuda").to(dtype) / 8
        for renorm in (True, False):
            check_route(logits, k, renorm=renorm, c=2.5)
    wide = torch.full((5, e + 11), 9.0, dtype=dtype, device="cuda")         # rows that start anywhere
    wide[:, 3:3 + e] = logits[:5]
    check_route(wide[:, 3:3 + e], k)


@gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("e,k,groups,top_groups,best", [(64, 6, 1, 1, 1), (16, 4, 4, 2, 2), (160, 6, 8, 3, 1), (256, 8, 8, 4, 2), (96, 8, 32, 5, 2),
                                                       (24, 8, 24, 7, 2), (1024, 8, 8, 2, 2), (30, 3, 5, 5, 1)])
def test_route_bias_and_groups(score, e, k, groups, top_groups, best):
    g = gen(e + groups)
    logits = torch.randint(-24, 25, (33, e), generator=g, device="cuda").float() / 8
    # multiples of 1/16 apart from the scores' own spacing; two experts in three share theirs, so that ties happen
    bias = torch.randint(-3, 4, (e,), generator=g, device="cuda").float() / 16
    check_route(logits, k, score=score, groups=groups, top_groups=top_groups, group_best=best, renorm=False)
    check_route(logits, k, score=score, bias=bias, groups=groups, top_groups=top_groups, group_best=best, c=0.5)
    flat = torch.zeros(e, device="cuda")
    check_route(logits, k, score=score, bias=flat, groups=groups, top_groups=top_groups, group_best=best)


@gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_route_masks(score, dtype):
    """Masked experts, rows that a mask leaves empty, the type's lowest value, infinities and NaN."""
    e, k, inf = 40, 6, float("inf")
    g = gen(5)
    logits = torch.randint(-30, 31, (12, e), generator=g, device="cuda").to(dtype) / 8
    logits[0] = -inf
    logits[1] = -inf
    logits[1, 7] = 1.0
    logits[2, ::2] = -inf
    logits[3] = torch.finfo(dtype).min
    logits[4, 5:] = torch.finfo(dtype).min
    logits[5, 11] = inf
    logits[6, 3] = float("nan")
    logits[7] = float("nan")
    logits[8, :] = -inf
    logits[8, 20:24] = 0.5
    logits[9] = 0.0
    logits[9, 1::2] = -0.0                                   # equal to +0
    check_route(logits, k, score=score)
    check_route(logits, k, score=score, renorm=False)
    got, _, _ = call_route(logits, k, score=score, groups=8, top_groups=2)
    want, gate, _ = route64(logits, k, score, None, 8, 2, 1, True, 1.0)
    assert torch.equal(got.cpu(), want)
    bias = torch.zeros(e, device="cuda")
    bias[::3] = -inf
    bias[1] = float("nan")
    finite = logits[[2, 9, 10, 11]].contiguous()
    check_route(finite, k, score=score, bias=bias)
    d = torch.empty_like(logits)
    idx, _, _ = call_route(logits, k, score=score)
    ops.moe_ovl_route_backward(logits=logits, expert=idx, dgate=torch.randn((12, k), generator=g, device="cuda"), dlogits=d, score=ops.SCORES[score])
    assert bool(d.isfinite().all()) and not d[0].any() and not d[7].any() and not d[2, ::2].any()


@gpu
def test_route_many_rows_and_optional_outputs():
    g = gen(2)
    logits = torch.randn((20011, 72), generator=g, device="cuda")
    i, gt, n = call_route(logits, 5, renorm=False)
    want = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :5]
    assert torch.equal(i.long(), want)
    p = torch.softmax(logits.double(), 1).gather(1, want)
    close(gt, p, 1e-5 * p)
    assert torch.equal(n.long(), torch.bincount(want.flatten(), minlength=72))
    i2, g2, _ = call_route(logits, 5, renorm=False, counts=False)
    assert torch.equal(i, i2) and torch.equal(gt, g2)
    n.fill_(4)
    ops.moe_ovl_route(logits=logits[:0], expert=i[:0], gate=gt[:0], counts=n)
    assert not n.any()


def route_backward64(logits, expert, dgate, score, renorm, c):
    z = logits.double().detach().requires_grad_()
    p = torch.softmax(z, 1) if score == "softmax" else torch.sigmoid(z)
    at = expert.long().clamp_min(0)
    live = (expert >= 0).double()
    s = p.gather(1, at) * live
    w = c * (s / s.sum(1, keepdim=True) if renorm else s)
    (w * dgate.double()).sum().backward()
    s, p, d = s.detach(), p.detach(), (dgate.double() * c).abs()
    # what the error is measured against: the magnitudes of the terms that are subtracted (and, for the 64-bit values' own
    # rounding, of those that cancel to 0 in them)
    total = s.sum(1, keepdim=True)
    if renorm:
        s = s / total
    dot = (d * s).sum(1, keepdim=True)
    size = (p if score == "softmax" and not renorm else 1e-9 * p / total) * dot
    return z.grad, size.scatter_add(1, at, s * (d + dot))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward(dtype, score, renorm):
    for e, k, rows in ((1, 1, 3), (8, 2, 70), (17, 5, 9), (64, 6, 1203), (130, 8, 33), (256, 8, 40), (384, 4, 5), (1000, 32, 7)):
        g = gen(e)
        logits = normal(g, (rows, e + 5), dtype, 1.5)[:, 2:2 + e] if e % 2 == 0 else normal(g, (rows, e), dtype, 1.5)
        expert, _, _ = call_route(logits, k, score=score, renorm=renorm)
        if k > 2:
            expert[0, k - 1] = -1
        dgate = torch.randn((rows, k), generator=g, device="cuda")
        out, full = guarded(rows, e, dtype, 3, 1)
        ops.moe_ovl_route_backward(logits=logits, expert=expert, dgate=dgate, dlogits=out, score=ops.SCORES[score], renormalise=renorm, gate_scale=1.5)
        want, size = route_backward64(logits, expert, dgate, score, renorm, 1.5)
        close(out, want, U[dtype] * want.abs() + 1e-5 * size + 1e-37)
        assert untouched(full, out)
        same = logits.clone()
        apart = torch.empty_like(same)
        for z, o in ((same, apart), (same, same)):
            ops.moe_ovl_route_backward(logits=z, expert=expert, dgate=dgate, dlogits=o, score=ops.SCORES[score], renormalise=renorm, gate_scale=1.5)
        assert torch.equal(same, apart)


@gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_backward_against_differences(score, renorm):
    g = gen(9)
    rows, e, k = 6, 40, 5
    logits = torch.randn((rows, e), generator=g, device="cuda")
    expert, _, _ = call_route(logits, k, score=score, renorm=renorm)
    dgate = torch.randn((rows, k), generator=g, device="cuda")
    out = torch.empty_like(logits)
    ops.moe_ovl_route_backward(logits=logits, expert=expert, dgate=dgate, dlogits=out, score=ops.SCORES[score], renormalise=renorm)

    def loss(z):
        s = (torch.softmax(z, 1) if score == "softmax" else torch.sigmoid(z)).gather(1, expert.long())
        return float(((s / s.sum(1, keepdim=True) if renorm else s) * dgate.double()).sum())

    for _ in range(4):
        v = torch.randn((rows, e), generator=g, device="cuda", dtype=torch.float64)
        num = (loss(logits.double() + 1e-5 * v) - loss(logits.double() - 1e-5 * v)) / 2e-5
        assert abs(num - float((out.double() * v).sum())) <= 1e-5 * float((out.double() * v).abs().sum())


# ------------------------------------------------------------------------------------------------ 8-bit product

def make8(g, shape, pad=0):
    full = torch.randint(-128, 128, (*shape[:-1], shape[-1] + pad), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    return full[..., :shape[-1]]


def product64(a, sa, b, sb, counts=None):
    if counts is None:
        b2, s2 = (b, sb) if b.dim() == 2 else (b[0], sb[0])
        return (a.double() @ b2.double().t()) * sa.double()[:, None] * s2.double()
    out, lo = torch.zeros((a.shape[0], b.shape[1]), dtype=torch.float64, device="cuda"), 0
    for e, c in enumerate(counts):
        hi = min(lo + max(c, 0), a.shape[0])
        out[lo:hi] = (a[lo:hi].double() @ b[e].double().t()) * sa[lo:hi].double()[:, None] * sb[e].double()
        lo = hi
    return out


def check_product(a, sa, b, sb, dtype, counts=None, pad=0, shift=0):
    """The integer sum is exact; its conversion, two products and the last rounding are what is left."""
    m, n = a.shape[0], b.shape[-2]
    out, full = guarded(m, n, dtype, pad, shift)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    dev_counts = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    ops.moe_ovl_quant_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=out, expert_counts=dev_counts, status=status)
    want = product64(a, sa, b, sb, counts)
    covered = m if counts is None else min(m, sum(max(c, 0) for c in counts))
    close(out[:covered], want[:covered], (U[dtype] + 3.1 * 2.0 ** -24) * want[:covered].abs() + FLOOR[dtype])
    assert untouched(full, out) and not status.any()
    if covered < m:
        assert bool((out[covered:].float() == 7.5).all())


SHAPES = [(1, 1, 16), (1, 5, 48), (2, 127, 128), (3, 128, 144), (16, 129, 256), (17, 300, 400), (31, 64, 1024), (33, 257, 2048), (64, 1000, 512), (65, 130, 272),
          (127, 256, 640), (128, 512, 4096), (129, 384, 1280), (200, 77, 16), (257, 513, 1040), (500, 2050, 2064), (1025, 768, 528), (1, 4096, 14336),
          (2000, 1500, 400), (4097, 640, 256)]


@gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_quant_matmul(m, n, k, dtype):
    g = gen(m + n)
    a, b = make8(g, (m, k), 32 if m % 3 == 0 else 0), make8(g, (n, k), 16 if n % 3 == 0 else 0)
    sa, sb = torch.rand(m, generator=g, device="cuda") * 1e-3, torch.rand(n, generator=g, device="cuda") * 1e-2
    check_product(a, sa, b, sb, dtype, pad=5 if m % 2 else 0, shift=1 if n % 2 else 0)


@gpu
def test_quant_matmul_longest_sums():
    """All -128: the largest sum that 32 bits hold, and signs that cancel."""
    k = ops.MAX_QUANT_K
    a = torch.full((3, k), -128, dtype=torch.int8, device="cuda")
    b = torch.full((130, k), -128, dtype=torch.int8, device="cuda")
    b[1] = 127
    b[2, ::2] = 127
    one = torch.ones(3, device="cuda")
    check_product(a, one, b, torch.ones(130, device="cuda"), F32)


@gpu
@pytest.mark.parametrize("counts,n,k", [([5], 130, 256), ([0, 3, 0], 256, 128), ([1] * 40, 96, 272), ([0, 0, 0, 17], 128, 512), ([100, 1, 0, 33, 250], 640, 1024),
                                        ([700, 300, 0, 513], 300, 208), ([3, 0, 2] * 30, 384, 640), ([1000] * 5, 512, 512), ([0] * 1023 + [7], 16, 64),
                                        ([2] * 700, 24, 48)])
def test_quant_matmul_experts(counts, n, k):
    m, e = sum(counts), len(counts)
    g = gen(m + n)
    a, b = make8(g, (m, k)), make8(g, (e, n, k))
    sa, sb = torch.rand(m, generator=g, device="cuda") * 1e-3, torch.rand((e, n), generator=g, device="cuda")
    check_product(a, sa, b, sb, BF16, counts)
    check_product(a, sa, b, sb, F32, counts, pad=3)


@gpu
def test_quant_matmul_counts_that_do_not_add_up():
    g = gen(4)
    a, b = make8(g, (90, 256)), make8(g, (4, 140, 256))
    sa, sb = torch.rand(90, generator=g, device="cuda"), torch.rand((4, 140), generator=g, device="cuda")
    check_product(a, sa, b, sb, F32, [20, 0, 30, 11])            # rows 61.. are left as they were
    check_product(a, sa, b, sb, F32, [50, 60, 70, 2147483647])   # cut at 90
    check_product(a, sa, b, sb, F32, [2147483647] * 4)
    check_product(a, sa, b, sb, F32, [-5, 40, -2147483648, 10])  # negative: none
    check_product(a, sa, b, sb, F32, [0, 0, 0, 0])


@gpu
def test_quant_matmul_scales_of_every_kind():
    a = torch.ones((4, 32), dtype=torch.int8, device="cuda")
    b = torch.ones((3, 32), dtype=torch.int8, device="cuda")
    b[2] = 0
    sa = torch.tensor([1.0, 0.0, float("inf"), float("nan")], device="cuda")
    out, status = torch.empty((4, 3), device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ops.moe_ovl_quant_matmul(a=a, a_scale=sa, b=b, b_scale=torch.tensor([1.0, -2.0, 1.0], device="cuda"), out=out, status=status)
    assert out[0].tolist() == [32.0, -64.0, 0.0] and not out[1].any()
    assert out[2, 0] == float("inf") and out[2, 1] == float("-inf") and bool(out[2, 2].isnan()) and bool(out[3].isnan().all())


@gpu
def test_quant_matmul_bounded_waits_run_out():
    """Test hook: no tile is loaded.  Every wait gives up, the status says so, and the next call on a cleared status is right."""
    g = gen(8)
    for m, n, k, counts in ((3, 1000, 2048, None), (700, 1024, 512, None), (300, 512, 512, [100, 0, 200]), (20, 256, 512, [10, 10])):
        e = 1 if counts is None else len(counts)
        a, b = make8(g, (m, k)), make8(g, (e, n, k))
        sa, sb = torch.rand(m, generator=g, device="cuda"), torch.rand((e, n), generator=g, device="cuda")
        out, status = torch.empty((m, n), dtype=BF16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
        dc = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        ops.moe_ovl_quant_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=out, status=status, expert_counts=dc, wait_timeout_us=3000,
                                 flags=ops.FLAG_QUANT_MATMUL_TEST_NO_LOADS)
        torch.cuda.synchronize()
        assert int(status[0]) == B.ERR_TIMEOUT
        check_product(a, sa, b, sb, BF16, counts)


# ------------------------------------------------------------------------------------------------ what they share

@gpu
def test_offsets_beyond_32_bits():
    """Rows that lie so far apart that element and byte offsets pass 32 bits."""
    g = gen(6)
    far, d = 1_500_000_016, 256

    def spread(rows, cols, dtype, src=None):
        full = torch.empty(far * (rows - 1) + cols, dtype=dtype, device="cuda")
        v = full.as_strided((rows, cols), (far, 1))
        if src is not None:
            v.copy_(src)
        return v

    x = spread(3, d, BF16, normal(g, (3, d), BF16))
    w = normal(g, (d,), BF16)
    q, scale = spread(3, d, torch.int8), torch.empty(3, device="cuda")
    ops.moe_ovl_add_norm(x=x, weight=w, q=q, scale=scale)
    v, _ = norm64(x, w, 1e-6)
    step = v.abs().amax(1, keepdim=True) / 127
    close(q.double() * scale.double()[:, None], v, 0.502 * step)
    b = make8(g, (200, d))
    out, status = spread(3, 200, BF16), torch.zeros(4, dtype=torch.int32, device="cuda")
    sb = torch.rand(200, generator=g, device="cuda")
    ops.moe_ovl_quant_matmul(a=q, a_scale=scale, b=b, b_scale=sb, out=out, status=status)
    want = product64(q, scale, b, sb)
    close(out, want, (U[BF16] + 2e-7) * want.abs() + 1e-38)
    logits = spread(3, 64, F32, torch.randint(-40, 41, (3, 64), generator=g, device="cuda").float())
    check_route(logits, 6)
    del x, out, logits
    gate_up = spread(3, 2 * d, BF16, normal(g, (3, 2 * d), BF16))
    ops.moe_ovl_swiglu_quant(gate_up=gate_up, q=q, scale=scale)
    a, c = gate_up[:, :d].double(), gate_up[:, d:].double()
    v = a * torch.sigmoid(a) * c
    close(q.double() * scale.double()[:, None], v, 0.502 * v.abs().amax(1, keepdim=True) / 127)


@gpu
def test_streams_and_graph_capture():
    """All operators on another stream, and captured once and replayed with new inputs: the same bits as direct calls."""
    g = gen(7)
    t, d, f, e, k = 70, 512, 256, 16, 2
    x, w, wg = normal(g, (t, d), BF16), normal(g, (d,), BF16), normal(g, (t, e), F32)
    b, sb = make8(g, (e, 2 * f, d)), torch.rand((e, 2 * f), generator=g, device="cuda") * 1e-3

    class Buffers:
        def __init__(s):
            s.y, s.q, s.scale, s.rstd = torch.zeros_like(x), torch.zeros((t, d), dtype=torch.int8, device="cuda"), torch.zeros(t, device="cuda"), torch.zeros(t, device="cuda")
            s.expert, s.gate, s.counts = torch.zeros((t, k), dtype=torch.int32, device="cuda"), torch.zeros((t, k), device="cuda"), torch.zeros(e, dtype=torch.int32, device="cuda")
            s.dl, s.dx, s.dw = torch.zeros_like(wg), torch.zeros_like(x), torch.zeros(d, device="cuda")
            s.out, s.status = torch.zeros((t, 2 * f), dtype=BF16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
            s.q2, s.scale2 = torch.zeros((t, f), dtype=torch.int8, device="cuda"), torch.zeros(t, device="cuda")
            s.ws = torch.zeros(ops.moe_ovl_add_norm_workspace_bytes(t, d), dtype=torch.uint8, device="cuda")
            s.rows = torch.tensor([t // e] * (e - 1) + [t - t // e * (e - 1)], dtype=torch.int32, device="cuda")

        def run(s, x, logits, stream=None):
            ops.moe_ovl_add_norm(x=x, weight=w, y=s.y, q=s.q, scale=s.scale, rstd=s.rstd, stream=stream)
            ops.moe_ovl_route(logits=logits, expert=s.expert, gate=s.gate, counts=s.counts, stream=stream)
            ops.moe_ovl_route_backward(logits=logits, expert=s.expert, dgate=s.gate, dlogits=s.dl, stream=stream)
            ops.moe_ovl_quant_matmul(a=s.q, a_scale=s.scale, b=b, b_scale=sb, out=s.out, expert_counts=s.rows, status=s.status, stream=stream)
            ops.moe_ovl_swiglu_quant(gate_up=s.out, q=s.q2, scale=s.scale2, stream=stream)
            ops.moe_ovl_add_norm_backward(dy=s.y, h=x, weight=w, rstd=s.rstd, dx=s.dx, dweight=s.dw, workspace=s.ws, stream=stream)

        def all(s):
            return (s.y, s.q, s.scale, s.rstd, s.expert, s.gate, s.counts, s.dl, s.dx, s.dw, s.out, s.q2, s.scale2)

    direct, other, captured = Buffers(), Buffers(), Buffers()
    direct.run(x, wg)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other.run(x, wg, stream=side)
    side.synchronize()
    for p, q in zip(direct.all(), other.all()):
        assert torch.equal(p, q)
    sx, sl = torch.zeros_like(x), torch.zeros_like(wg)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run(sx, sl)
    for _ in range(2):
        x = normal(g, (t, d), BF16)
        wg = normal(g, (t, e), F32)
        sx.copy_(x)
        sl.copy_(wg)
        graph.replay()
        direct.run(x, wg)
        for p, q in zip(direct.all(), captured.all()):
            assert torch.equal(p, q)


@gpu
def test_one_behind_the_other():
    """Every operator reads what the one in front wrote, back to back: the same bits as with a synchronize after each call.  The
    shapes take the kernels by turns that start early and late, short and long ones; buffers are written again in the next turn while
    the one before it may still be ending."""
    g = gen(31)
    shapes = [(1, 512, 256), (40, 512, 256), (3000, 512, 256), (300, 2048, 1408), (20000, 512, 384)]
    scale = lambda *shape: torch.full(shape, 1 / (74 * shape[-1] ** 0.5), device="cuda")  # noqa: E731  outputs of about 1: 74 is the weights' rms
    weights = [(1 + normal(g, (d,), BF16, 0.1), make8(g, (8, 2 * f, d)), scale(8, 2 * f, d)[..., 0].contiguous(), make8(g, (8, d, f)),
                scale(8, d, f)[..., 0].contiguous(), normal(g, (t, d), BF16)) for t, d, f in shapes]

    def run(sync):
        outs = []
        for (t, d, f), (w, b1, s1, b2, s2, x0) in zip(shapes, weights):
            new = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
            x, y, dx, dw = x0.clone(), new(t, d), new(t, d), new(d, dtype=F32)
            q, qs, rstd = new(t, d, dtype=torch.int8), new(t, dtype=F32), new(t, dtype=F32)
            h, q2, qs2 = new(t, 2 * f), new(t, f, dtype=torch.int8), new(t, dtype=F32)
            expert, gate, counts = new(t, 1, dtype=torch.int32), new(t, 1, dtype=F32), new(8, dtype=torch.int32)
            dl, status = new(t, 8), new(4, dtype=torch.int32)
            ws = torch.zeros(max(16, ops.moe_ovl_add_norm_workspace_bytes(t, d)), dtype=torch.uint8, device="cuda")
            logits = y[:, :8]
            calls = [
                lambda: ops.moe_ovl_add_norm(x=x, residual=dx, residual_out=x, weight=w, y=y, q=q, scale=qs, rstd=rstd),
                lambda: ops.moe_ovl_route(logits=logits, expert=expert, gate=gate, counts=counts, renormalise=False),
                lambda: ops.moe_ovl_quant_matmul(a=q, a_scale=qs, b=b1, b_scale=s1, out=h, expert_counts=counts, status=status),
                lambda: ops.moe_ovl_swiglu_quant(gate_up=h, q=q2, scale=qs2),
                lambda: ops.moe_ovl_quant_matmul(a=q2, a_scale=qs2, b=b2, b_scale=s2, out=y, expert_counts=counts, status=status),
                lambda: ops.moe_ovl_route_backward(logits=logits, expert=expert, dgate=gate, dlogits=dl, renormalise=False),
                lambda: ops.moe_ovl_add_norm_backward(dy=y, h=x, weight=w, rstd=rstd, dx=dx, dweight=dw, workspace=ws),
            ]
            torch.cuda.synchronize()
            for _ in range(6):
                for c in calls:
                    c()
                    if sync:
                        torch.cuda.synchronize()
            torch.cuda.synchronize()
            assert not status.any() and int(counts.sum()) == t
            outs += [x, y, dx, dw, q, qs, rstd, h, q2, qs2, expert, gate, counts, dl]
        return outs

    for n, (a, b) in enumerate(zip(run(True), run(False))):
        assert torch.equal(torch.nan_to_num(a.float(), nan=-77.0), torch.nan_to_num(b.float(), nan=-77.0)), n


@gpu
def test_product_does_not_count_the_time_of_what_is_in_front():
    """Its waits are bounded from its own start: with a limit of 150 us behind 2 GB of gated activation, at least 2.1e9 / 8e12 s = 260 us."""
    g = gen(32)
    f = 4096
    x = torch.ones((131072, 2 * f), dtype=BF16, device="cuda")
    q, s = torch.empty((131072, f), dtype=torch.int8, device="cuda"), torch.empty(131072, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    for m in (5, 300, 2048):
        a, b = make8(g, (m, 512)), make8(g, (1024, 512))
        sa, sb = torch.rand(m, generator=g, device="cuda"), torch.rand(1024, generator=g, device="cuda")
        want, out = torch.empty((m, 1024), dtype=BF16, device="cuda"), torch.empty((m, 1024), dtype=BF16, device="cuda")
        ops.moe_ovl_quant_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=want, status=status)
        torch.cuda.synchronize()
        ops.moe_ovl_swiglu_quant(gate_up=x, q=q, scale=s)
        ops.moe_ovl_quant_matmul(a=a, a_scale=sa, b=b, b_scale=sb, out=out, status=status, wait_timeout_us=150)
        torch.cuda.synchronize()
        assert not status.any() and torch.equal(out, want)


@gpu
def test_tensors_that_do_not_fit_are_refused():
    x, w = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.ones(64, dtype=BF16, device="cuda")
    q, s = torch.zeros((4, 64), dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    st = torch.zeros(4, dtype=torch.int32, device="cuda")
    i, gt = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    out = torch.zeros((4, 32), dtype=BF16, device="cuda")
    b, sb = torch.zeros((32, 64), dtype=torch.int8, device="cuda"), torch.zeros(32, device="cuda")
    norm, bwd, swi, rt, rtb, mm = (ops.moe_ovl_add_norm, ops.moe_ovl_add_norm_backward, ops.moe_ovl_swiglu_quant, ops.moe_ovl_route,
                                   ops.moe_ovl_route_backward, ops.moe_ovl_quant_matmul)
    E = torch.zeros((2, 32, 64), dtype=torch.int8, device="cuda")
    wrong = [
        (norm, dict(x=x, weight=w.float()[:32])), (norm, dict(x=x, weight=w.half())), (norm, dict(x=x.int(), weight=w)), (norm, dict(x=x.t(), weight=w[:4])),
        (norm, dict(x=x, weight=w, q=q)), (norm, dict(x=x, weight=w, q=q, scale=s[:2])), (norm, dict(x=x, weight=w, y=x[:2])), (norm, dict(x=x, weight=w, eps=-1.0)),
        (norm, dict(x=x, weight=w, residual=x.float())), (norm, dict(x=x, weight=w, eps=float("nan"))), (norm, dict(x=x.cpu(), weight=w)),
        (norm, dict(x=x[:1].expand(4, 64), weight=w)), (norm, dict(x=x[0], weight=w)), (norm, dict(x=x, weight=w.cpu())),
        (bwd, dict(dy=x, h=x[:3], weight=w, rstd=s, dx=x)), (bwd, dict(dy=x, h=x, weight=w, rstd=s[:2], dx=x)),
        (swi, dict(gate_up=x[:, :63], q=q[:, :31], scale=s)), (swi, dict(gate_up=x, q=q, scale=s)),
        (rt, dict(logits=x, expert=i.long(), gate=gt)), (rt, dict(logits=x, expert=i, gate=gt[:2])), (rt, dict(logits=x, expert=i, gate=gt, num_groups=5)),
        (rt, dict(logits=x, expert=i, gate=gt, num_groups=4, top_groups=5)), (rt, dict(logits=x, expert=i, gate=gt, group_best=3)), (rt, dict(logits=x[:, :1], expert=i, gate=gt)),
        (rt, dict(logits=x, expert=i, gate=gt, bias=s)), (rt, dict(logits=x, expert=i, gate=gt, counts=st)), (rt, dict(logits=x, expert=i, gate=gt, score=2)),
        (rt, dict(logits=x, expert=i, gate=gt, gate_scale=float("nan"))),
        (rtb, dict(logits=x, expert=i, dgate=gt, dlogits=x.float())), (rtb, dict(logits=x, expert=i, dgate=gt[:1], dlogits=x)),
        (mm, dict(a=q, a_scale=s, b=b, b_scale=sb, out=out[:, :16], status=st)), (mm, dict(a=q, a_scale=s, b=b[:, :32], b_scale=sb, out=out, status=st)),
        (mm, dict(a=q, a_scale=s[:2], b=b, b_scale=sb, out=out, status=st)), (mm, dict(a=q, a_scale=s, b=b, b_scale=sb[:3], out=out, status=st)),
        (mm, dict(a=q, a_scale=s, b=E, b_scale=sb, out=out, status=st)), (mm, dict(a=q, a_scale=s, b=b, b_scale=sb, out=out, status=st, expert_counts=st)),
        (mm, dict(a=q, a_scale=s, b=b, b_scale=sb, out=out.int(), status=st)), (mm, dict(a=q, a_scale=s, b=b, b_scale=sb, out=out, status=st[:2])),
        (mm, dict(a=q, a_scale=s, b=b, b_scale=sb, out=out, status=st, flags=8)),
    ]
    for n, (f, kw) in enumerate(wrong):
        with pytest.raises(B.MoeOvlError) as err:
            f(**kw)
        assert err.value.code == B.ERR_INVALID_ARG, n
    unsupported = [
        (norm, dict(x=torch.zeros((1, 32769), device="cuda"), weight=torch.zeros(32769, device="cuda"))),
        (mm, dict(a=q[:, :40], a_scale=s, b=b[:, :40], b_scale=sb, out=out, status=st)),        # k not a multiple of 16
        (mm, dict(a=q[:, 8:56], a_scale=s, b=b[:, :48], b_scale=sb, out=out, status=st)),       # starts off a multiple of 16
        (rt, dict(logits=torch.zeros((2, 1025), device="cuda"), expert=i[:2], gate=gt[:2])),
        (rt, dict(logits=x, expert=torch.zeros((4, 33), dtype=torch.int32, device="cuda"), gate=torch.zeros((4, 33), device="cuda"))),
        (rt, dict(logits=x, expert=i, gate=gt, num_groups=64)),
    ]
    for n, (f, kw) in enumerate(unsupported):
        with pytest.raises(B.MoeOvlError) as err:
            f(**kw)
        assert err.value.code == B.ERR_UNSUPPORTED, n
    dw = torch.zeros(64, device="cuda")
    for ws in (None, torch.zeros(64 * 4 * 4 - 4, dtype=torch.uint8, device="cuda")):
        with pytest.raises(B.MoeOvlError) as err:
            bwd(dy=x, h=x, weight=w, rstd=s, dx=x, dweight=dw, workspace=ws)
        assert err.value.code == B.ERR_WORKSPACE
    torch.cuda.synchronize()


def test_host_side_refusals():
    """What the C side refuses before it touches a device: no GPU needed.  The pointers are never followed."""
    lib = B.load()
    for name in ("moe_ovl_add_norm", "moe_ovl_add_norm_backward", "moe_ovl_swiglu_quant", "moe_ovl_route", "moe_ovl_route_backward", "moe_ovl_quant_matmul"):
        assert getattr(lib, name)(None) == B.ERR_INVALID_ARG
    P = 0x10000

    def norm(**kw):
        a = ops.NormArgs(struct_size=ctypes.sizeof(ops.NormArgs), device=0, rows=4, d=64, dtype=0, weight_dtype=0, eps=1e-6, x=P, weight=P, x_stride=64)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.moe_ovl_add_norm(ctypes.byref(a))

    for kw in (dict(struct_size=8), dict(rows=-1), dict(d=0), dict(dtype=3), dict(weight_dtype=1), dict(x=None), dict(x=P + 1), dict(q=P), dict(scale=P),
               dict(x_stride=63), dict(x_stride=-64), dict(flags=1), dict(device=-1), dict(eps=-1.0), dict(residual=P, residual_stride=3)):
        assert norm(**kw) == B.ERR_INVALID_ARG, kw
    assert norm(d=40000, x_stride=40000) == B.ERR_UNSUPPORTED

    def mm(**kw):
        a = ops.QuantMatmulArgs(struct_size=ctypes.sizeof(ops.QuantMatmulArgs), rows=4, n=32, k=64, out_dtype=0, a=P, a_scale=P, b=P, b_scale=P, out=P, status=P,
                                a_stride=64, b_stride=64, out_stride=32)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.moe_ovl_quant_matmul(ctypes.byref(a))

    for kw in (dict(struct_size=8), dict(rows=-1), dict(n=0), dict(k=0), dict(num_experts=-1), dict(num_experts=2), dict(expert_counts=P), dict(flags=2), dict(a=None),
               dict(status=None), dict(out_stride=31), dict(a_stride=48), dict(out_dtype=7), dict(wait_timeout_us=-1)):
        assert mm(**kw) == B.ERR_INVALID_ARG, kw
    for kw in (dict(k=60), dict(k=131072, a_stride=131072, b_stride=131072), dict(num_experts=1025, expert_counts=P), dict(a=P + 8), dict(b_stride=72),
               dict(num_experts=1000, expert_counts=P, n=1 << 30)):
        assert mm(**kw) == B.ERR_UNSUPPORTED, kw
    x = torch.zeros((4, 64))
    with pytest.raises(B.MoeOvlError) as err:
        ops.moe_ovl_add_norm(x=x, weight=torch.zeros(64))
    assert err.value.code == B.ERR_INVALID_ARG
    n = ops.moe_ovl_add_norm_workspace_bytes(5, 64)
    assert n == 5 * 64 * 4 and ops.moe_ovl_add_norm_workspace_bytes(10 ** 6, 64) == 888 * 64 * 4
