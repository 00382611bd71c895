"""Values at which the operators that make a worker's gradient could go wrong: NaN and infinities where they must come
through, the ends of a type's range, padding, row shapes between the usual ones, and bounds that hold their precision."""
import copy
import math
import pickle

import pytest
import torch

from paper_1905_10936_b200 import binding as ef
from paper_1905_10936_b200 import build as efbuild
from paper_1905_10936_b200 import ops
from test_ops_gpu import (EPS, F8, TYPES, U, act64, check_policy, gen, ids, policy64, policy_case, quantised, randn, rounded, slope64,
                          strided, values_of, within)


pytestmark = pytest.mark.gpu


@pytest.fixture
def wait_limit():
    """Sets the attempts after which the operators' waits on the device give up (checked build)."""
    ef.use_library(efbuild.build_library(debug=True))
    try:
        yield ef.ef_debug_wait_limit
    finally:
        torch.cuda.synchronize()
        ef.ef_debug_wait_limit(-1)
        ef.use_library(None)


# ---- policy loss -----------------------------------------------------------------------------
SPECIAL = [(name, value) for name in ("old", "adv", "ref") for value in (math.nan, math.inf, -math.inf)]


@pytest.mark.parametrize("with_ref", [True, False], ids=["kl", "no kl"])
@pytest.mark.parametrize("n,c", [(40, 300), (320, 4000), (40, 20000)])
def test_policy_loss_passes_on_what_is_not_finite(n, c, with_ref):
    """NaN and infinities among a live row's scalars reach its loss and gradient as in the formulas (a NaN on either side of
    the minimum is the minimum), and no other row's.  Rows of one warp, of four, of eight."""
    lo, hi, beta = 0.2, 0.28, 0.1
    x, t, old, adv, w, ref = policy_case(c, n, c, torch.float32, masked=0.0)
    x[x == -math.inf] = -9.0
    use = dict(clip_low=lo, clip_high=hi, beta=beta)
    good = ops.policy_loss(x, t, old, adv, w, ref_logp=ref if with_ref else None, **use)
    v = {"old": old.clone(), "adv": adv.clone(), "ref": ref.clone()}
    special = SPECIAL if with_ref else SPECIAL[:6]
    for i, (name, value) in enumerate(special):
        v[name][3 * i] = value
    i = 3 * len(special)                                          # a target of probability 0 that the old policy never gave either
    x2 = x.clone()
    x2[i, t[i]] = -math.inf
    v["old"][i] = -math.inf
    v["adv"][i + 1] = 0.0                                         # an infinite ratio times nothing
    v["old"][i + 1] = -math.inf
    out = ops.policy_loss(x2, t, v["old"], v["adv"], w, ref_logp=v["ref"] if with_ref else None, **use)
    e = policy64(x2, t, v["old"], v["adv"], w, v["ref"] if with_ref else None, lo, hi, beta, 1.0)
    coef = torch.where(e["straight"].isnan() | e["lp"].isnan(), torch.full_like(e["coef"], math.nan), e["coef"])
    special_rows = torch.zeros(n, dtype=torch.bool, device="cuda")
    special_rows[[3 * k for k in range(len(special) + 1)] + [i + 1]] = True
    assert torch.equal(out.grad[~special_rows], good.grad[~special_rows])
    assert torch.equal(out.token_loss[~special_rows], good.token_loss[~special_rows])
    tok = e["tok"]
    for k in special_rows.nonzero().view(-1).tolist():
        assert bool(tok[k].isnan() == out.token_loss[k].isnan()) and bool(tok[k].isinf() == out.token_loss[k].isinf()), k
        if bool(coef[k].isnan()):
            assert bool(out.grad[k].isnan().all()), k
        elif bool(coef[k].isinf()):
            assert not bool(out.grad[k].isfinite().any()), k
        else:
            want = -coef[k] * e["p"][k]
            want[t[k]] += coef[k]
            within(out.grad[k], want, 1e-5 * coef[k].abs() + 1e-37, f"grad of row {k}")
    assert bool(out.loss.isnan())


def test_policy_loss_of_many_long_rows_passes_on_what_is_not_finite():
    """The same, by the kernel of many long rows: which rows are NaN, infinite and finite is as with few rows."""
    n, c = 320, 20000
    x, t, old, adv, w, ref = policy_case(c, n, c, torch.float32, masked=0.0)
    for i, (name, value) in enumerate(SPECIAL):
        {"old": old, "adv": adv, "ref": ref}[name][3 * i] = value
    many = ops.policy_loss(x, t, old, adv, w, ref_logp=ref, beta=0.1)
    few = ops.policy_loss(x[:40], t[:40], old[:40], adv[:40], w[:40], ref_logp=ref[:40], beta=0.1)
    for a, b in ((many.token_loss[:40], few.token_loss), (many.grad[:40], few.grad)):
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.isinf(), b.isinf())
    assert bool(many.token_loss[40:].isfinite().all()) and bool(many.grad[40:].isfinite().all()) and bool(many.loss.isnan())


@pytest.mark.parametrize("need_grad", [True, False], ids=["gradient", "loss only"])
def test_many_of_the_longest_rows_repeat_bit_for_bit(need_grad):
    """Three rows and more per CTA, each loaded over the one before while that is still read: whichever CTA takes a row, and
    however far its warps are apart, the row's result has the same bits."""
    n, c = 900, 50257
    x, t, old, adv, w, ref = policy_case(2, n, c, torch.bfloat16)
    call = lambda: ops.policy_loss(x, t, old, adv, w, ref_logp=ref, beta=0.04, need_grad=need_grad)  # noqa: E731
    first = call()
    e = policy64(x, t, old, adv, w, ref, 0.2, 0.2, 0.04, 1.0)
    within(first.logp, e["logp"], 1e-5, "logp")
    for _ in range(6):
        again = call()
        assert torch.equal(again.logp, first.logp) and torch.equal(again.token_loss, first.token_loss)
        assert not need_grad or torch.equal(again.grad, first.grad)


@pytest.mark.parametrize("n,c,dtype", [(1500, 301, torch.bfloat16), (320, 4000, torch.float32), (9, 50257, torch.float32),
                                       (3, 300001, torch.bfloat16), (450, 13001, torch.bfloat16), (900, 50257, torch.bfloat16)], ids=str)
def test_policy_rows_whose_waits_run_out_are_nan(n, c, dtype, wait_limit):
    """Waits that give up at once, or after a few attempts: the call ends, a row is right or NaN as a whole, the loss is NaN if a
    row is, and the next call is right again.  Rows of one and four warps, of eight in clusters, many long ones."""
    x, t, old, adv, w, ref = policy_case(c, n, c, dtype)
    x[x == -math.inf] = -9.0
    live = w != 0
    for need_grad in (True, False):
        call = lambda: ops.policy_loss(x, t, old, adv, w, ref_logp=ref, beta=0.04, need_grad=need_grad)  # noqa: E731
        good = call()
        assert bool(good.token_loss.isfinite().all())
        for attempts in (0, 1, 3, 20):
            wait_limit(attempts)
            for _ in range(3):
                out = call()
                lost = out.logp.isnan()
                assert torch.equal(out.token_loss.isnan(), lost)
                assert torch.equal(out.logp[~lost], good.logp[~lost]) and torch.equal(out.token_loss[~lost], good.token_loss[~lost])
                assert bool(out.loss.isnan()) == bool(lost.any())
                if need_grad:
                    assert bool(out.grad[lost].isnan().all()) and torch.equal(out.grad[~lost], good.grad[~lost])
                assert attempts > 0 or bool(lost[live].all())
        wait_limit(-1)
        again = call()
        assert torch.equal(again.logp, good.logp) and torch.equal(again.loss, good.loss)


@pytest.mark.parametrize("c,dtype", [(12288, torch.bfloat16), (12289, torch.bfloat16), (6144, torch.float32), (6145, torch.float32),
                                     (53248, torch.bfloat16), (53249, torch.bfloat16), (26624, torch.float32), (26625, torch.float32),
                                     (53248, torch.float16)], ids=str)
def test_policy_loss_on_both_sides_of_the_many_rows_borders(c, dtype):
    """Enough rows for the kernels of four warps and of resident CTAs to be chosen, up to the widest row of which two share an
    SM, and the next wider one.  logp's bound: its own rounding (u |logp|), the target's distance from the maximum (u of it), 4 u
    for the exponentials' approximation and 2 u for their sum."""
    n = 310
    x, t, old, adv, w, ref = policy_case(c, n, c, dtype)
    e = policy64(x, t, old, adv, w, ref, 0.2, 0.28, 0.04, 1.0)
    e["t"] = t
    depth = e["x"].amax(dim=1) - e["x"].gather(1, t[:, None]).view(n)
    for view in (x, strided(x, 3, 1)):
        for place in (False, True):
            xv = strided(x, 3, 1) if place and view is not x else x.clone()
            out = ops.policy_loss(xv, t, old, adv, w, ref_logp=ref, clip_low=0.2, clip_high=0.28, beta=0.04, in_place=place)
            check_policy(out, e, dtype, 0.04, 1.0, adv, old, ref)
            within(out.logp, e["logp"], U * (e["lp"].abs() + depth + 6.0), "logp")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=ids)
def test_log_probabilities_and_loss_of_a_whole_vocabulary(dtype):
    """50257 logits, many rows and few.  logp as above.  A token's loss before its own rounding is off by that of the ratio's
    exponent (as logp, without the rounding of logp itself: 6 u and the distance), of expf (4 u) and six more roundings, times ratio
    and advantage; the KL term's slope is below 0.1; the clipped side has three roundings and its own size."""
    n, c = 600, 50257
    x, t, old, adv, w, ref = policy_case(7, n, c, dtype)
    e = policy64(x, t, old, adv, w, ref, 0.2, 0.2, 0.04, 1.0)
    depth = e["x"].amax(dim=1) - e["x"].gather(1, t[:, None]).view(n)
    for rows in (n, 40):
        within(ops.token_logprob(x[:rows], t[:rows]), e["lp"][:rows], (U * (e["lp"].abs() + depth + 6.0))[:rows], "logp")
    out = ops.policy_loss(x, t, old, adv, w, ref_logp=ref, beta=0.04)
    off = U * (depth + 16.0) * (e["straight"].abs() + 0.1) * w.to(F8) + 4 * U * e["tok"].abs()
    within(out.token_loss, e["tok"], off, "token loss")
    total = e["tok"].sum()
    within(out.loss[None], total[None], off.sum() + U * total.abs(), "loss")


# ---- weight gradient -------------------------------------------------------------------------
@pytest.mark.parametrize("n,c,j,dtype", [(65, 129, 257, torch.bfloat16), (2085, 1001, 777, torch.float32), (8192, 512, 1024, torch.bfloat16),
                                         (1500, 300, 100, torch.float16)], ids=str)
def test_weight_gradients_whose_waits_run_out_are_nan(n, c, j, dtype, wait_limit):
    """Waits that give up at once, or after a few attempts: the call ends, a value is right or NaN, and the next call is right again."""
    kept, dy = ops.checkpoint_save(randn(n, n, c)), randn(n + 1, n, j, dtype=dtype)
    good = ops.checkpoint_weight_grad(kept, dy)
    assert bool(good.isfinite().all())
    for attempts in (0, 1, 3, 20):
        wait_limit(attempts)
        for _ in range(3):
            out = ops.checkpoint_weight_grad(kept, dy)
            assert bool(((out == good) | out.isnan()).all())
            assert attempts > 0 or bool(out.isnan().all())
    wait_limit(-1)
    assert torch.equal(ops.checkpoint_weight_grad(kept, dy), good)


@pytest.mark.parametrize("n", [16, 64, 576, 2085])
def test_weight_grad_of_few_fp32_gradients_is_as_near_as_an_fp32_product(n):
    """2-norm distance from 64 bits, next to that of the same product in fp32, whose sums are rounded at each step."""
    kept, dy = ops.checkpoint_save(randn(1, n, 256)), randn(2, n, 200)
    x = values_of(kept)
    want, plain = x.t() @ dy.to(F8), x.float().t() @ dy
    got = ops.checkpoint_weight_grad(kept, dy)
    assert float((got.to(F8) - want).norm()) <= float((plain.to(F8) - want).norm())


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("n,c,j", [(8192, 384, 640), (9000, 1000, 130)])
def test_weight_grad_keeps_the_precision_of_an_fp32_product(n, c, j, dtype):
    """The tensor core cuts its running sum, so one accumulator over all tokens is 4e-6 off in the 2-norm and grows with their
    number; in spans of 18 stages that are added up in registers the error is that of an fp32 product, 3e-7, twice of which is allowed."""
    kept, dy = ops.checkpoint_save(randn(1, n, c)), randn(2, n, j, dtype=dtype)
    want = values_of(kept).t() @ dy.to(F8)
    got = ops.checkpoint_weight_grad(kept, dy)
    assert float((got.to(F8) - want).norm()) <= 6e-7 * float(want.norm())


# ---- checkpoints -----------------------------------------------------------------------------
def test_fp16_values_stay_finite_in_a_checkpoint():
    """Every finite fp16 value next to any other: what the checkpoint stands for is finite in fp16, at most one step off where
    the nearest code would not be and half a step elsewhere, and the operators' fp16 outputs with it."""
    top = torch.finfo(torch.float16).max
    x = torch.zeros(4, 256, dtype=torch.float16, device="cuda")
    x[0] = torch.linspace(-top, top, 256, device="cuda").half()
    x[1, 0], x[1, 1], x[1, 2], x[1, 3] = top, -top, 65024.0, 64992.0
    x[1, 130], x[1, 131] = 65024.0, -65024.0                      # a group whose largest has code 127 of scale 512
    x[2, :128] = -top                                             # a mask
    x[3, 255] = 65056.0
    for view in (x, strided(x, 5, 3), x[:, :251]):
        kept = ops.checkpoint_save(view)
        back = ops.checkpoint_load(kept, torch.float16)
        assert bool(back.isfinite().all())
        assert torch.equal(back.to(F8), values_of(kept))          # no rounding of the values themselves
        step = kept.scales.to(F8).repeat_interleave(128, dim=1)[:, :view.shape[1]]
        high = view.to(F8).abs() >= 65024.0
        off = (values_of(kept) - view.to(F8)).abs()
        assert bool((off <= torch.where(high, 1.0, 0.5) * step).all())
        assert torch.equal(values_of(kept)[~high], quantised(view)[~high])
    assert torch.equal(ops.checkpoint_load(ops.checkpoint_save(x), torch.float16)[1, 130:132], x[1, 130:132])
    out = ops.activation_forward(x, "gelu", checkpoint_out=True)
    assert bool(out.a.isfinite().all())
    out = ops.activation_forward(torch.cat([x, torch.ones_like(x)], dim=1), "swiglu", checkpoint_out=True)
    assert bool(out.a.isfinite().all())
    # outputs are computed in fp32: those that round to a finite fp16 value stay finite, others are infinite as they would be without codes
    h = torch.zeros(2, 200, dtype=torch.float16, device="cuda")
    h[:, 0] = 1.0
    w = torch.zeros(200, device="cuda")
    scale = math.sqrt(200.0)
    w[0] = 65519.0 / scale * (1 - 1e-6)
    y = ops.rmsnorm_forward(h, w, 0.0, checkpoint=True).y
    assert bool(y.isfinite().all()) and float(y[0, 0]) == 64512.0
    w[0] = 70000.0 / scale
    plain, kept = ops.rmsnorm_forward(h, w, 0.0), ops.rmsnorm_forward(h, w, 0.0, checkpoint=True)
    assert plain.y[0, 0] == math.inf and kept.y[0, 0] == math.inf
    # fp32 and bf16 hold 65536: their checkpoints are as before
    for dtype in (torch.float32, torch.bfloat16):
        z = torch.full((1, 8), 65500.0, device="cuda").to(dtype)
        assert bool((ops.checkpoint_load(ops.checkpoint_save(z), dtype) == 65536.0).all())


@pytest.mark.parametrize("own", [False, True], ids=["one buffer", "two tensors"])
def test_copies_of_a_checkpoint_outlive_it(own):
    x = randn(1, 70, 300)
    kept = ops.checkpoint_save(x)
    if own:
        kept = ops.Checkpoint(kept.codes.clone(), kept.scales.clone(), 300)
    want, grad = ops.checkpoint_load(kept), ops.checkpoint_weight_grad(kept, x)
    others = [copy.deepcopy(kept), pickle.loads(pickle.dumps(kept))]
    kept.codes.fill_(77)
    kept.scales.fill_(1.0)
    for other in others:
        assert torch.equal(ops.checkpoint_load(other), want) and torch.equal(ops.checkpoint_weight_grad(other, x), grad)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("c", [1, 300, 1001, 1004])
def test_norm_leaves_the_codes_behind_a_row_zero(c, dtype):
    """Also where rstd is NaN or infinite, which times the nothing behind the row's end is NaN."""
    x = torch.ones(4, c, dtype=dtype, device="cuda")
    x[0, c // 2], x[1, c - 1], x[2] = math.nan, math.inf, 0.0
    out = ops.rmsnorm_forward(x, torch.ones(c, device="cuda"), 0.0, checkpoint=True)
    assert bool(out.rstd[0].isnan()) and out.rstd[2] == math.inf
    assert not bool(out.checkpoint.codes[:, c:].any())
    assert bool(out.y[0].isnan().all()) and bool(out.y[2].isnan().all()) and not bool(out.y[3].isnan().any())


# ---- activation ------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids)
@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
def test_activation_slope_far_out(kind, dtype):
    """The slope of a large input is that of the asymptote, as far as a checkpoint's values reach."""
    big = torch.tensor([1e3, 1e10, 1.7e19, 2e19, 1e25, 1e38, 127 * 2.0 ** 121], device="cuda")
    c = 128 * len(big)
    z = torch.zeros(2, c, device="cuda")
    z[0, ::128], z[1, ::128] = big, -big
    z = z.to(dtype)
    if kind == "swiglu":
        z = torch.cat([z, torch.ones_like(z)], dim=1)
    out = ops.activation_forward(z, kind)
    dz = ops.activation_backward(torch.ones(2, c, device="cuda", dtype=dtype), out.z, kind)[:, :c:128]
    assert bool((dz[0] == 1.0).all()) and bool((dz[1] == 0.0).all())


@pytest.mark.parametrize("kind", ["gelu", "swiglu"])
def test_activation_is_as_near_in_fp32_as_elementary_operations(kind):
    """2-norm distance from 64 bits of a and dz, next to that of the same formulas in elementary fp32 operations, each of
    which is rounded once.  A quarter more is allowed."""
    n, c = 64, 4096
    parts = 2 if kind == "swiglu" else 1
    z, da = randn(1, n, c * parts, scale=2.0), randn(2, n, c)
    out = ops.activation_forward(z, kind)
    got = ops.activation_backward(da, out.z, kind).view(n * parts, c)
    zq = values_of(out.z)
    d, _ = slope64(zq, kind)
    up = da.repeat_interleave(parts, dim=0)
    want_a, want = act64(zq, kind, c), up.to(F8) * d
    q = zq.float()
    if kind == "gelu":
        v = math.sqrt(2.0 / math.pi) * (q + 0.044715 * q * q * q)
        th = torch.tanh(v)
        a = 0.5 * q * (1.0 + th)
        slope = 0.5 * (1.0 + th) + 0.5 * q * (1.0 - th * th) * math.sqrt(2.0 / math.pi) * (1.0 + 3.0 * 0.044715 * q * q)
    else:
        g, u = q[0::2], q[1::2]
        s = torch.sigmoid(g)
        a, slope = g * s * u, torch.empty_like(q)
        slope[0::2], slope[1::2] = u * s * (1.0 + g * (1.0 - s)), g * s
    for what, mine, plain, exact in (("a", out.a, a, want_a), ("dz", got, up * slope, want)):
        off, ref = float((mine.to(F8) - exact).norm()), float((plain.to(F8) - exact).norm())
        assert off <= 1.25 * ref, (what, off, ref)


# ---- norm ------------------------------------------------------------------------------------
@pytest.mark.parametrize("c", [7, 1000, 1603, 4096])
def test_norm_rstd_is_rounded_once(c):
    """Whole numbers whose squares add up to less than 2^24: the sum is exact, so rstd is the rounded 64-bit value."""
    n = 500
    x = torch.randint(-40, 41, (n, c), device="cuda", generator=gen(c)).float()
    x[torch.arange(n, device="cuda"), torch.arange(n, device="cuda") % c] = 2000.0
    want = 1.0 / torch.sqrt((x.to(F8) ** 2).mean(dim=1) + float(torch.tensor(EPS)))
    assert float((x.to(F8) ** 2).sum(dim=1).max()) < 2.0 ** 24
    assert torch.equal(ops.rmsnorm_forward(x, torch.ones(c, device="cuda"), EPS).rstd, want.float())


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("c", [513, 600, 768, 1025, 1280, 1536, 2049, 2560, 2900, 5120, 6144, 6145])
def test_norm_of_rows_between_the_powers_of_two(c, dtype):
    """Rows of 3, 6, 12 and 24 warps, and of 12 warps with two segments each (fp32), have launch shapes of their own.  Bounds as
    in the tests of the other widths: an error of (n + 64) u of the summed magnitudes for dw, of 84 u for dx, 48 u for y."""
    for n in (1, 700):
        x, r = randn(c, n, c, dtype=dtype, scale=2.0), randn(c + 1, n, c, dtype=dtype)
        dy, dh, w = randn(c + 2, n, c, dtype=dtype), randn(c + 3, n, c, dtype=dtype), 1.0 + 0.2 * randn(c + 4, c)
        for view in (lambda t: t, lambda t: strided(t, 5, 3)):
            out = ops.rmsnorm_forward(view(x), w, EPS, residual=view(r), checkpoint=True)
            h = x.to(F8) + r.to(F8)
            rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + EPS)
            y = h * rstd[:, None] * w.to(F8)
            within(out.h, h, rounded(h, dtype, U * h.abs()), "h")
            within(out.rstd, rstd, 48 * U * rstd, "rstd")
            step = out.checkpoint.scales.to(F8).repeat_interleave(128, dim=1)[:, :c]
            within(values_of(out.checkpoint), y, 0.5 * step + 96 * U * y.abs(), "codes")
            kept = ops.checkpoint_save(x)
            for source, hv in ((view(x), x.to(F8)), (kept, values_of(kept))):
                got, got_w = ops.rmsnorm_backward(view(dy), source, w, out.rstd, dh=view(dh))
                nh, uv = hv * out.rstd.to(F8)[:, None], dy.to(F8) * w.to(F8)
                dot = (uv * nh).mean(dim=1, keepdim=True)
                dx = out.rstd.to(F8)[:, None] * (uv - nh * dot) + dh.to(F8)
                size = out.rstd.to(F8)[:, None] * (uv.abs() + nh.abs() * (uv * nh).abs().mean(dim=1, keepdim=True))
                within(got, dx, rounded(dx, dtype, 84 * U * size + U * dh.to(F8).abs()), "dx")
                within(got_w, (dy.to(F8) * nh).sum(dim=0), (n + 64) * U * (dy.to(F8) * nh).abs().sum(dim=0), "dw")


# ---- tensors that torch differentiates -------------------------------------------------------
def test_leaves_that_require_gradients_are_not_overwritten():
    x, t, old, adv, w, _ = policy_case(1, 5, 40, torch.float32)
    leaf = x.clone().requires_grad_()
    for bad in (leaf, leaf[1:4]):
        k = bad.shape[0]
        with pytest.raises(ValueError, match="requires gradients"):
            ops.policy_loss(bad, t[:k], old[:k], adv[:k], w[:k], in_place=True)
    assert torch.equal(leaf.detach(), x)
    ops.policy_loss(leaf, t, old, adv, w)                         # read only
    ops.policy_loss(leaf, t, old, adv, w, need_grad=False, in_place=True)
    kept, dy = ops.checkpoint_save(x.nan_to_num(neginf=0.0)), torch.ones(5, 8, device="cuda")
    weight = torch.zeros(40, 8, device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="requires gradients"):
        ops.checkpoint_weight_grad(kept, dy, out=weight)
    assert not bool(weight.detach().any())
    with torch.no_grad():
        ops.checkpoint_weight_grad(kept, dy, out=weight)
        ops.policy_loss(leaf, t, old, adv, w, in_place=True)
    base = torch.zeros(3, 40, requires_grad=True, device="cuda")  # logits of a model, whose backward pass does not need them
    logits = base * 2.0 + x[:3].nan_to_num(neginf=-9.0)
    out = ops.policy_loss(logits, t[:3], old[:3], adv[:3], w[:3], in_place=True)
    logits.backward(out.grad)
    assert torch.equal(base.grad, 2.0 * out.grad)
