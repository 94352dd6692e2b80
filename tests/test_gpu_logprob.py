"""Log-probabilities over a vocabulary and their gradient on the GPU, against the definition in 64 bits.

Bounds are element by element, from the arithmetic: a product of bf16 numbers is exact in fp32, a sum of K of them in fp32
is off by at most K 2^-24 of the sum of their magnitudes (fp32 inputs: six such sums, and 2^-23 of a term is left out),
an fp32 function by 2^-22 of its value or argument, a rounding to bf16 by 2^-8 of the value.
"""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(n, h, v, dtype, seed, per_row=None, sigma=2.0):
    """Inputs on the CPU: X, W, tgt_ptr, tgt, dlogp; per_row: targets of each row (default 0 to 3 of them)."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, h), generator=g).to(DT[dtype])
    w = (torch.randn((v, h), generator=g) * sigma / h ** 0.5).to(DT[dtype])
    k = torch.randint(0, 4, (n,), generator=g) if per_row is None else torch.tensor(per_row)
    ptr = torch.cat([torch.zeros(1, dtype=torch.long), k.cumsum(0)]).int()
    e = int(ptr[-1])
    tgt = torch.randint(0, v, (e,), generator=g).int()
    return x, w, ptr, tgt, torch.randn(e, generator=g)


def reference(x, w, ptr, tgt, dlogp, scale):
    """The definition in 64 bits, and bounds on what fp32 sums and the roundings of the type may be off by."""
    fp32 = x.dtype == torch.float32
    x, w, g = x.double(), w.double(), dlogp.double()
    n, h = x.shape
    v = w.shape[0]
    left_out = 2.0 ** -23 if fp32 else 0.0
    half = U if fp32 else 2.0 ** -8
    sums = 6 if fp32 else 1                      # products of planes per product
    z = scale * x @ w.t()
    zerr = scale * ((sums * h + 4) * U + left_out) * (x.abs() @ w.abs().t())
    lse = torch.logsumexp(z, 1) if n else torch.zeros(0, dtype=torch.float64)
    # a lane's chain of 64 terms, 7 exchanges, its tiles (at most v / 8192), the rescaling; arguments and results of exp2 and log2
    chain = 64 + 7 + 4 + v // 8192
    lerr = zerr.amax(1) + (chain + 4) * U + 8 * U * (z.abs().amax(1) + lse.abs()) if n else lse
    logp, perr = torch.zeros(tgt.numel(), dtype=torch.float64), torch.zeros(tgt.numel(), dtype=torch.float64)
    dz, dzerr = torch.zeros_like(z), torch.zeros_like(z)
    live = torch.zeros(n, dtype=torch.bool)
    for r in range(n):
        total, mags = 0.0, 0.0
        for e in range(int(ptr[r]), int(ptr[r + 1])):
            t = int(tgt[e])
            if not 0 <= t < v:
                continue
            logp[e] = z[r, t] - lse[r]
            perr[e] = zerr[r, t] + lerr[r] + 2 * U * (z[r, t].abs() + lse[r].abs())
            total, mags = total + float(g[e]), mags + abs(float(g[e]))
            dz[r, t] += g[e]
            dzerr[r, t] += 4 * U * mags
            live[r] = live[r] or g[e] != 0
        p = torch.exp(z[r] - lse[r])
        dz[r] -= total * p
        perr_r = zerr[r] + lerr[r] + 16 * U * (z[r].abs() + lse[r].abs() + 1)
        dzerr[r] += abs(total) * p * torch.expm1(perr_r) + 8 * U * mags * p
    dz[~live] = 0
    dzerr[~live] = 0
    x = torch.where(live[:, None], x, torch.zeros((), dtype=torch.float64))
    dz, dzerr = scale * dz, scale * dzerr
    dzerr = dzerr + (half + 4 * U) * (dz.abs() + dzerr)
    da = dz.abs() + dzerr
    dx, dw = dz @ w, dz.t() @ x
    dxerr = dzerr @ w.abs() + ((sums * v + 16) * U + left_out) * (da @ w.abs())
    dwerr = dzerr.t() @ x.abs() + ((sums * n + 16) * U + left_out) * (da.t() @ x.abs())
    out = dict(logp=logp, LSE=lse, dX=dx, dW=dw)
    err = dict(logp=perr, LSE=lerr, dX=dxerr + half * (dx.abs() + dxerr), dW=dwerr + half * (dw.abs() + dwerr))
    return out, {k: e + 1e-37 for k, e in err.items()}


def call(x, w, ptr, tgt, dlogp, scale=1.0):
    from paper_2608_25683_amd import psattn as P
    x, w, ptr, tgt, dlogp = (t.cuda() for t in (x, w, ptr, tgt, dlogp))
    logp, lse = P.psattn_logprob_fwd(x, w, ptr, tgt, logit_scale=scale)
    dx, dw = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, dlogp, logit_scale=scale)
    torch.cuda.synchronize()
    return dict(logp=logp, LSE=lse, dX=dx, dW=dw)


def check(got, ref, err, what):
    for k, r in ref.items():
        d = (got[k].double().cpu() - r).abs()
        bad = ~(d <= err[k])
        worst = float((d / err[k]).max()) if d.numel() else 0.0
        print(f"{what} {k}: {worst:.3f} of the bound", file=sys.stderr, flush=True)
        assert not bad.any(), f"{k}: {int(bad.sum())} of {bad.numel()} elements, worst {worst:.3g} of the bound"


# from one element to several tiles of every size the kernels use (32, 128 and 256 rows, 128 and 256 entries), odd ones among
# them, with the summed dimension short of a stage, a stage and one more element, and split over workgroups (dX: vocabularies
# above 512 behind few rows; dW: many rows before few entries)
SHAPES = [(1, 8, 1), (1, 64, 7), (2, 72, 300), (63, 128, 129), (64, 8, 128), (65, 136, 257), (130, 264, 1001), (257, 64, 2500),
          (300, 192, 515), (9, 520, 4100), (520, 256, 770),
          (32, 64, 640), (33, 1032, 385), (1500, 16, 140), (5, 2056, 96)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,h,v", SHAPES)
def test_against_the_definition(n, h, v, dtype):
    a = make(n, h, v, dtype, 100 * n + v)
    scale = 1.0 if n % 2 else 1.25
    check(call(*a, scale=scale), *reference(*a, scale), f"{dtype} {n}x{h}x{v}")


@pytest.mark.parametrize("dtype,n", [("bf16", 257), ("bf16", 320), ("bf16", 321), ("bf16", 590), ("bf16", 64), ("fp32", 129), ("fp32", 192),
                                     ("fp32", 193), ("fp32", 300), ("fp32", 61)])
def test_last_rows_before_a_large_vocabulary(dtype, n):
    """Up to 64 rows behind the whole tiles of 256 (fp32: 128) have narrow ones; one row more, and these are whole too."""
    a = make(n, 72, 24001, dtype, n, per_row=[1] * n)
    check(call(*a), *reference(*a, 1.0), f"{dtype} {n}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_targets_and_targets_left_out(dtype):
    n, h, v = 70, 64, 300
    x, w, ptr, tgt, g = make(n, h, v, dtype, 7, per_row=[0, 5, 1, 0, 2] * 14)
    tgt[::4] = -100
    tgt[1::7] = v                     # just behind the vocabulary
    tgt[2] = 2 ** 31 - 1
    tgt[int(ptr[6]):int(ptr[7])] = 11  # the same target five times
    g[3::5] = 0
    a = (x, w, ptr, tgt, g)
    got = call(*a)
    check(got, *reference(*a, 1.0), dtype)
    assert torch.all(got["logp"].cpu()[(tgt < 0) | (tgt >= v)] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_without_gradient_do_not_reach_others(dtype):
    """Infinities and NaN in rows that no adjoint enters: their own gradient is 0, the others' are as without them."""
    n, h, v = 150, 72, 400
    x, w, ptr, tgt, g = make(n, h, v, dtype, 8, per_row=[1, 2, 0] * 50)
    dead = torch.zeros(n, dtype=torch.bool)
    dead[2::3] = True
    for r in (0, 40, 148):             # rows whose adjoints are zero
        g[int(ptr[r]):int(ptr[r + 1])] = 0
        dead[r] = True
    clean = call(x, w, ptr, tgt, g)
    y = x.clone()
    y[dead] = float("nan")
    y[2, ::2] = float("inf")
    got = call(y, w, ptr, tgt, g)
    assert torch.equal(got["dW"], clean["dW"]) and torch.all(got["dX"][dead.cuda()] == 0)
    assert torch.equal(got["dX"], clean["dX"])
    assert torch.equal(got["LSE"].cpu()[~dead], clean["LSE"].cpu()[~dead])
    assert torch.isnan(got["LSE"].cpu()[dead]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,alive", [(256, 0.3), (257, 0.9), (1000, 0.02), (2500, 0.5), (777, 0.0)])
def test_few_rows_with_a_gradient(n, alive, dtype):
    """The live rows are packed for the products, each 256 rows by themselves: any share of them, in blocks and scattered."""
    g = torch.Generator().manual_seed(n)
    k = (torch.rand(n, generator=g) < alive).long() * torch.randint(1, 3, (n,), generator=g)
    k[n // 3:n // 2] = 0
    a = make(n, 72, 300, dtype, n, per_row=k.tolist())
    a[4][::5] = 0
    got = call(*a)
    check(got, *reference(*a, 1.0), f"{dtype} {n} rows, {alive} alive")
    assert not got["dX"][(k == 0).cuda()].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_rows_no_targets(dtype):
    from paper_2608_25683_amd import psattn as P
    x, w, ptr, tgt, g = make(0, 64, 100, dtype, 1, per_row=[])
    got = call(x, w, ptr, tgt, g)
    assert got["logp"].numel() == 0 and got["LSE"].numel() == 0 and got["dX"].shape == (0, 64) and not got["dW"].any()
    a = make(5, 64, 100, dtype, 1, per_row=[0] * 5)
    got = call(*a)
    check(got, *reference(*a, 1.0), dtype)
    assert not got["dX"].any() and not got["dW"].any()
    dx, dw = P.psattn_logprob_bwd(*(t.cuda() for t in a[:4]), got["LSE"], a[4].cuda(), need_dX=False)
    assert dx is None and not dw.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_gradient_alone_is_the_same(dtype):
    from paper_2608_25683_amd import psattn as P
    x, w, ptr, tgt, g = (t.cuda() for t in make(140, 128, 700, dtype, 9))
    _, lse = P.psattn_logprob_fwd(x, w, ptr, tgt)
    dx, dw = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, g)
    a, b = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, g, need_dW=False)
    assert b is None and torch.equal(a, dx)
    a, b = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, g, need_dX=False)
    assert a is None and torch.equal(b, dw)


def test_one_token_is_the_target_of_all_rows():
    """More targets in one tile than its list holds at a time, and rows with hundreds of targets."""
    n, h, v = 4500, 64, 300
    x, w, ptr, tgt, g = make(n, h, v, "bf16", 61, per_row=[1] * n)
    tgt[:] = 77
    tgt[::1000] = 299
    got = call(x, w, ptr, tgt, g)
    xd, wd, gd = x.double(), w.double(), g.double()
    z = xd @ wd.t()
    p = torch.softmax(z, 1)
    dz = -gd[:, None] * p
    dz[torch.arange(n), tgt.long()] += gd
    # dz and the results are rounded once each (uniform in a binade: 2^-8.8 in the mean square at most)
    for name, ref in (("dX", dz @ wd), ("dW", dz.t() @ xd)):
        rel = float((got[name].double().cpu() - ref).norm() / ref.norm())
        assert rel <= 2 * 2.0 ** -8.8, (name, rel)
    a = make(7, h, v, "bf16", 62, per_row=[0, 700, 1, 0, 333, 2, 900])
    check(call(*a), *reference(*a, 1.0), "hundreds of targets")


def test_rounding_of_a_targets_dz_does_not_reach_the_gradients():
    """The dz of a row's target is most of it; its rounding to bf16 alone would be 2^-9.8 of dX in the mean square beside the
    result's own, sqrt(2) of that together.  What it leaves out is added, so the whole error stays within 1.15 of the result's
    own rounding, measured on the exact result."""
    x, w, ptr, tgt, g = make(512, 256, 3000, "bf16", 71, per_row=[1] * 512)
    got = call(x, w, ptr, tgt, g)
    xd, wd, gd = x.cuda().double(), w.cuda().double(), g.cuda().double()
    dz = -gd[:, None] * torch.softmax(xd @ wd.t(), 1)
    dz[torch.arange(512, device="cuda"), tgt.cuda().long()] += gd
    for name, ref in (("dX", dz @ wd), ("dW", dz.t() @ xd)):
        own = float((ref.bfloat16().double() - ref).norm())
        assert float((got[name].double() - ref).norm()) <= 1.15 * own, name


def test_confident_rows():
    """p near 1: the target's dz is dlogp (1 - p), formed before it is rounded; and logits far apart."""
    for sigma, boost in ((2.0, 4.0), (30.0, 0.0)):
        x, w, ptr, tgt, g = make(80, 128, 500, "bf16", 21, per_row=[1] * 80, sigma=sigma)
        x = (x.float() + boost * w[tgt.long()].float()).bfloat16()
        a = (x, w, ptr, tgt, g)
        check(call(*a), *reference(*a, 1.0), f"sigma {sigma}")


def test_targets_listed_in_any_way():
    """tgt_ptr outside 0 .. targets, or descending, is taken as the nearest value that is not: nothing is read outside."""
    from paper_2608_25683_amd import psattn as P
    x, w, _, _, _ = make(4, 64, 50, "bf16", 3, per_row=[1] * 4)
    tgt = torch.tensor([3, 4, 5], dtype=torch.int32)
    bad = torch.tensor([-5, 2, 1, 99, 2 ** 31 - 1], dtype=torch.int32)      # rows: [0, 2), [2, 2), [1, 3), [3, 3)
    logp, lse = P.psattn_logprob_fwd(x.cuda(), w.cuda(), bad.cuda(), tgt.cuda())
    z = x.double() @ w.double().t()
    z = z - torch.logsumexp(z, 1)[:, None]
    assert abs(float(logp[0]) - float(z[0, 3])) < 1e-4 and abs(float(logp[2]) - float(z[2, 5])) < 1e-4


@pytest.mark.parametrize("n,h,v", [(8200, 64, 40001), (20003, 72, 30011)])
def test_several_pieces_of_the_vocabulary(n, h, v):
    """Sizes at which the backward takes more than one piece (at most 512 MiB of dz), by the definition on the GPU in 64 bits."""
    for dtype in ("bf16", "fp32"):
        x, w, ptr, tgt, g = make(n, h, v, dtype, 5)
        got = call(x, w, ptr, tgt, g)
        xd, wd = x.cuda().double(), w.cuda().double()
        z = xd @ wd.t()
        lse = torch.logsumexp(z, 1)
        row = torch.repeat_interleave(torch.arange(n), (ptr[1:] - ptr[:-1]).long()).cuda()
        t, gd = tgt.cuda().long(), g.cuda().double()
        logp = z[row, t] - lse[row]
        total = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, row, gd)
        dz = -total[:, None] * torch.exp(z - lse[:, None])
        dz.index_put_((row, t), gd, accumulate=True)
        for name, ref, tol in (("logp", logp, 2e-6), ("LSE", lse, 2e-6), ("dX", dz @ wd, None), ("dW", dz.t() @ xd, None)):
            rel = float((got[name].double() - ref).norm() / ref.norm())
            # gradients: dz and the result rounded once each (bf16: 2^-8 at most, uniform in a binade, so under 2^-8.8 in the
            # mean square, twice); fp32: sums of up to 6 x 40001 terms, random signs, 2^-24 x sqrt of that = 2.9e-5
            tol = tol or (2 * 2.0 ** -8.8 if dtype == "bf16" else 3e-5)
            print(f"{dtype} {n}x{h}x{v} {name}: rel {rel:.3g}", file=sys.stderr, flush=True)
            assert rel <= tol, (dtype, name, rel)


def test_repeats_bitwise_and_leaves_what_is_not_its_own():
    from paper_2608_25683_amd import psattn as P
    x, w, ptr, tgt, g = (t.cuda() for t in make(333, 136, 1030, "bf16", 31))
    room = lambda t, dt=torch.float32: torch.full((t + 64,), 7.0, dtype=dt, device="cuda")
    held = []
    for _ in range(3):
        logp, lse, dx, dw = room(tgt.numel()), room(333), room(x.numel(), x.dtype), room(w.numel(), x.dtype)
        ws = torch.full((P.psattn_logprob_workspace_size(333, tgt.numel(), 136, 1030, "bf16", 1) + 256,), 0xEE, dtype=torch.uint8, device="cuda")
        n = ws.numel() - 256
        P.psattn_logprob_fwd(x, w, ptr, tgt, logp=logp[:-64], LSE=lse[:-64], ws=ws[:n])
        P.psattn_logprob_bwd(x, w, ptr, tgt, lse[:-64], g, dX=dx[:-64].view_as(x), dW=dw[:-64].view_as(w), ws=ws[:n])
        assert torch.all(ws[n:] == 0xEE)
        for t in (logp, lse, dx, dw):
            assert torch.all(t[-64:] == 7.0)
        held.append([logp, lse, dx, dw])
    for other in held[1:]:
        assert all(torch.equal(a, b) for a, b in zip(held[0], other))


def test_on_another_stream_and_captured():
    from paper_2608_25683_amd import psattn as P
    args = [tuple(t.cuda() for t in make(200, 128, 900, "bf16", s, per_row=[1] * 200)) for s in (41, 42)]
    eager = [call(*a) for a in args]
    x, w, ptr, tgt, g = (t.clone() for t in args[0])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        logp, lse = P.psattn_logprob_fwd(x, w, ptr, tgt)
        dx, dw = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, g)
    s.synchronize()
    assert torch.equal(dx, eager[0]["dX"]) and torch.equal(dw, eager[0]["dW"]) and torch.equal(logp, eager[0]["logp"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logp, lse = P.psattn_logprob_fwd(x, w, ptr, tgt)
        dx, dw = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, g)
    for k in (0, 1, 1, 0):
        for dst, src in zip((x, w, ptr, tgt, g), args[k]):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        for name, t in (("logp", logp), ("LSE", lse), ("dX", dx), ("dW", dw)):
            assert torch.equal(t, eager[k][name]), (k, name)
        call(*args[1 - k])             # the program's own work between the replays


def test_weights_beyond_4_gib():
    """70001 x 32768 bf16: offsets that pass 32 bits.  Only some rows of W are non-zero, so that the rest is known: those logits are 0."""
    from paper_2608_25683_amd import psattn as P
    n, h, v, rows = 40, 32768, 70001, [0, 35000, 65535, 65536, 70000]
    g = torch.Generator().manual_seed(81)
    x = torch.randn((n, h), generator=g).bfloat16()
    some = (torch.randn((len(rows), h), generator=g) * 2 / h ** 0.5).bfloat16()
    w = torch.zeros((v, h), dtype=torch.bfloat16, device="cuda")
    w[rows] = some.cuda()
    ptr, tgt = torch.arange(n + 1, dtype=torch.int32), torch.tensor([rows[r % 5] for r in range(n)], dtype=torch.int32)
    dlogp = torch.randn(n, generator=g)
    logp, lse = P.psattn_logprob_fwd(x.cuda(), w, ptr.cuda(), tgt.cuda())
    dx, dw = P.psattn_logprob_bwd(x.cuda(), w, ptr.cuda(), tgt.cuda(), lse, dlogp.cuda())
    z = x.double() @ some.double().t()
    ref = torch.log(torch.exp(z).sum(1) + (v - 5))
    pick = torch.arange(n) % 5
    # (5 logits of 32768 terms of about 1/90 each, and 70000 terms of the sum: well under 1e-4 in fp32)
    assert float((lse.double().cpu() - ref).abs().max()) <= 1e-4
    assert float((logp.double().cpu() - (z[torch.arange(n), pick] - ref)).abs().max()) <= 2e-4
    dz = -dlogp.double()[:, None] * torch.exp(z - ref[:, None])
    dz[torch.arange(n), pick] += dlogp.double()
    want = torch.cat([dz.t() @ x.double(), (-dlogp.double() * torch.exp(-ref))[None] @ x.double()])
    got = torch.cat([dw[rows].cpu(), dw[12345:12346].cpu()]).double()
    for a, b in ((got, want), (dx.double().cpu(), dz @ some.double())):
        assert float((a - b).norm() / b.norm()) <= 2.0 ** -8


def test_finite_differences():
    """dX and dW against central differences of the loss sum_e dlogp_e logp_e, fp32, through the forward alone."""
    from paper_2608_25683_amd import psattn as P
    x, w, ptr, tgt, g = (t.cuda() for t in make(6, 16, 40, "fp32", 51, per_row=[1, 2, 0, 1, 3, 1]))
    _, lse = P.psattn_logprob_fwd(x, w, ptr, tgt)
    dx, dw = P.psattn_logprob_bwd(x, w, ptr, tgt, lse, g)
    loss = lambda a, b: float((P.psattn_logprob_fwd(a, b, ptr, tgt)[0].double() * g.double()).sum())
    step = 2.0 ** -6
    # the difference's own error: step^2 / 6 of a third derivative (at most |dlogp| |other side|^3, here under 50) and two
    # losses off by 1e-6 of their terms
    tol = step ** 2 / 6 * 50 + 2e-6 * float(g.abs().sum()) * 5 / (2 * step)
    for which, grad in ((0, dx), (1, dw)):
        for idx in [(0, 0), (1, 5), (3, 15), (5, 7)]:
            lo, hi = [x.clone(), w.clone()], [x.clone(), w.clone()]
            lo[which][idx] -= step
            hi[which][idx] += step
            num = (loss(*hi) - loss(*lo)) / (2 * step)
            assert abs(num - float(grad[idx])) <= tol, (which, idx, num, float(grad[idx]))
