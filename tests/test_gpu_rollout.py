"""GPU parity of spec_top_logits, spec_distill_loss_fwd_bwd and
spec_verify_probs against the float64 oracle, through the C ABI."""

import numpy as np
import pytest
import torch

from paper_2606_12370_amd import binding
from tests.rollout_inputs import LOWEST, TYPES, check_distill, check_probs, check_top, lists, logit_rows, probs

pytestmark = pytest.mark.gpu
DT = ["f32", "bf16"]


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.load_library()
    yield
    torch.cuda.synchronize()


# ---- top logits --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("R,V,M", [(1, 1, 1), (3, 5, 4), (2, 7, 64), (5, 255, 256), (4, 256, 256), (7, 2049, 17),
                                   (3, 8191, 1), (2, 8192, 256), (3, 8193, 100), (5, 40001, 64), (1, 151936, 64),
                                   (1, 100003, 256), (300, 9001, 33), (1100, 4097, 20), (1500, 777, 256)])
def test_top_sizes(R, V, M, dtype):
    z = logit_rows((R, V), TYPES[dtype], 7 * R + V)
    check_top(binding.top_logits(z, M, 0.8), z, M, np.float32(0.8))


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("R", [2, 1100])
@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "two values", "sawtooth", "blocks"])
def test_top_orders(order, R, dtype):
    """Rows whose order makes every tile a candidate, and rows of ties."""
    V = 20000
    v = torch.arange(V, dtype=torch.float32)
    row = {"ascending": v * 0.01, "descending": -v * 0.01, "equal": torch.full((V,), -2.5),
           "two values": (v % 97 == 5).float(), "sawtooth": (v % 512) * 0.125 + v * 1e-5,
           "blocks": torch.floor(v / 700) % 7}[order]
    z = row.repeat(R, 1).to(TYPES[dtype]).cuda()
    for M in (1, 100, 256):
        out = binding.top_logits(z, M)
        check_top({k: t[:2] for k, t in out.items()}, z[:2], M, 1.0)
        for t in out.values():
            assert torch.equal(t, t[:1].expand_as(t))


@pytest.mark.parametrize("dtype", DT)
def test_top_masks_and_special_values(dtype):
    ty = TYPES[dtype]
    V, M = 9000, 40
    z = logit_rows((9, V), ty, 5)
    z[0] = -torch.inf
    z[1] = -torch.inf
    z[1, 8999] = 3.0
    z[2, ::3] = -torch.inf
    z[3, 30:] = LOWEST[ty]          # a mask of the lowest value: listed after the rest
    z[4] = LOWEST[ty]
    z[5, 4000] = torch.nan
    z[6, 8500] = torch.inf
    z[7] = 0.0
    z[7, 1::2] = -0.0               # one value: index order
    z[8, 60:] = -torch.inf
    out = binding.top_logits(z, M, 0.5)
    ref = check_top(out, z, M, 0.5)
    assert (ref["ids"][0] == -1).all() and (ref["ids"][5:7] == -1).all() and ref["ids"][1, 0] == 8999
    out = binding.top_logits(z, M, want_logz=False)
    check_top(out, z, M, 1.0, want_logz=False)


@pytest.mark.parametrize("dtype", DT)
def test_top_row_temperatures_and_strides(dtype):
    """The first K of K + 1 rows of a padded, offset tensor, a temperature a row."""
    big = logit_rows((6, 5, 5003), TYPES[dtype], 11)
    z = big[1:5, 1:4, 3:4999]
    T = torch.tensor([0.5, 1.0, 2.0, 0.9], device="cuda")
    check_top(binding.top_logits(z, 50, T), z, 50, T.cpu().numpy())
    one = logit_rows((1, 5003), TYPES[dtype], 12).expand(4, 5003)   # one row read four times
    check_top(binding.top_logits(one, 9, T), one, 9, T.cpu().numpy())
    bad = torch.tensor([0.5, 0.0, torch.nan, torch.inf], device="cuda")
    check_top(binding.top_logits(z, 50, bad), z, 50, bad.cpu().numpy())


@pytest.mark.parametrize("dtype", DT)
def test_top_extreme_temperatures(dtype):
    """Temperatures from the smallest float32 to the largest: 0 at T near 0 stays 0."""
    z = logit_rows((6, 5000), TYPES[dtype], 13)
    z[:, 0] = 0.0
    z[:2] = -z[:2].abs()
    T = torch.tensor([1.4e-45, 1e-38, 1e-20, 1e-3, 1e20, 3e38], device="cuda")
    out = binding.top_logits(z, 10, T)
    z64 = z.double()
    assert torch.equal(out["ids"][:, 0].long(), z64.argmax(-1))
    want = torch.logsumexp((z64 - z64.amax(-1, keepdim=True)) / T.double()[:, None], -1) + z64.amax(-1) / T.double()
    assert torch.allclose(out["logz"], want.float(), rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("scale", [1e3, 1e5, 1e30])
@pytest.mark.parametrize("dtype", DT)
def test_top_huge_logits(dtype, scale):
    """The product of a logit and log2(e) / T then has no fraction bits left."""
    z = (logit_rows((3, 5000), torch.float32, 14) * scale).to(TYPES[dtype])
    z[0] = z[0, 0]  # every term counts
    z[1] -= 10 * scale
    check_top(binding.top_logits(z, 20, 0.7), z, 20, np.float32(0.7))
    T = torch.tensor([0.3, 1.0, 7.0], device="cuda")
    check_top(binding.top_logits(z, 20, T), z, 20, T.cpu().numpy())


# ---- distillation --------------------------------------------------------------------

def run_distill(z, ids, val, lz, T=1.0, kind="forward", scale=0.75, grad_dtype=None):
    got = binding.distill_loss_fwd_bwd(z, ids, val, lz, temperature=T, kind=kind, scale=scale, grad_dtype=grad_dtype)
    fwd = binding.distill_loss_fwd_bwd(z, ids, val, lz, temperature=T, kind=kind, scale=scale, want_grad=False)
    torch.cuda.synchronize()
    assert fwd[2] is None
    check_distill(fwd, z, ids, val, lz, T, kind, scale)
    return got, check_distill(got, z, ids, val, lz, T, kind, scale)


@pytest.mark.parametrize("kind", ["forward", "ce"])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("N,K,V,M", [(1, 1, 1, 1), (2, 1, 5, 3), (3, 2, 7, 16), (2, 3, 1023, 256), (2, 8, 4097, 20),
                                     (3, 2, 16385, 64), (2, 2, 40001, 100), (1, 1, 151936, 64)])
def test_distill_sizes(N, K, V, M, dtype, tail, kind):
    z = logit_rows((N, K, V), TYPES[dtype], N + V)
    ids, val, lz = lists(N, K, V, M, 3 * V, T=0.8)
    for gd in ({torch.float32, TYPES[dtype]}):
        run_distill(z, ids, val, lz if tail else None, T=0.8, kind=kind, grad_dtype=gd)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T", [0.25, 1.0, 3.0])
def test_distill_student_near_the_teacher(dtype, T):
    """A student close to its teacher: a small loss between large terms, most of
    the mass on the list."""
    t = torch.randn((4, 2, 30000), generator=torch.Generator().manual_seed(9)) * 5.0
    ids, val, lz = lists(4, 2, 30000, 128, 0, T=T, near=t)
    z = (t + 0.05 * torch.randn(t.shape, generator=torch.Generator().manual_seed(10))).to(TYPES[dtype]).cuda()
    for x in (lz, None):
        run_distill(z, ids, val, x, T=T)


@pytest.mark.parametrize("dtype", DT)
def test_distill_lists(dtype):
    """Empty, padded, repeated, unsorted and covering lists, data errors."""
    ty = TYPES[dtype]
    N, K, V, M = 12, 2, 5000, 24
    z = logit_rows((N, K, V), ty, 21)
    ids, val, lz = lists(N, K, V, M, 22)
    ids[0] = -1                                # no entries
    ids[1, :, 5:] = -1                         # a short list, unused values arbitrary
    ids[2, :, ::2] = -7
    ids[3] = torch.flip(ids[3], (-1,))         # any order
    val[3] = torch.flip(val[3], (-1,))
    ids[4, 0, 10:] = ids[4, 0, 3]              # one id many times (values add up to more than 1 there:
    val[4, 0, 10:] -= 3.0                      # less mass than before)
    ids[5, 0, 3] = V                           # beyond the vocabulary
    val[5, 1, 3] = torch.nan
    ids[6, 0, 0] = -1
    val[6, 0, 0] = torch.nan                   # the mark of a data error, also in an unused entry
    val[6, 1, 0] = torch.inf
    val[7, 0, 4:] = -torch.inf                 # entries without probability
    val[7, 1] = -torch.inf
    lz[8, 0] = torch.nan
    lz[8, 1] = torch.inf
    lz[9, 0] -= 1.0                            # a log Z below the list's own: W > 1, no tail
    z[10, 0, 17] = torch.nan
    z[10, 1, 4000] = torch.inf
    z[11, 0] = -torch.inf
    z[0, 1] = torch.nan                        # not read: its list is empty
    for x in (lz, None):
        for kind in ("forward", "ce"):
            got, ref = run_distill(z, ids, val, x, kind=kind)
            bad = np.isnan(ref["per_step"])
            assert bad[5].all() and bad[6].all() and bad[10].all() and bad[11, 0] and not bad[:5].any()
            assert torch.isnan(got[0]).all()
            assert not got[2][0].any() and (got[1][0] == 0).all()


@pytest.mark.parametrize("dtype", DT)
def test_distill_masks(dtype):
    """Masked draft logits: listed ones make the loss infinite, unlisted ones have
    no gradient; masks of the lowest value; lists that hold the whole vocabulary or
    all of what the student allows."""
    ty = TYPES[dtype]
    N, V, M = 7, 6000, 60
    z = logit_rows((N, 1, V), ty, 31)
    ids, val, lz = lists(N, 1, V, M, 32)
    listed = torch.zeros((N, 1, V + 1), dtype=torch.bool, device="cuda")
    listed.scatter_(2, ids.long(), True)
    listed = listed[..., :V]
    z[0, 0, ids[0, 0, 3].long()] = -torch.inf
    z[1] = torch.where(listed[1], z[1], -torch.inf)        # no unlisted token has mass: the tail's loss is infinite
    z[2] = torch.where(listed[2], z[2], LOWEST[ty])
    z[3] = torch.where(listed[3], torch.full_like(z[3], -torch.inf), z[3])
    z[4] = LOWEST[ty]                                      # a flat row
    z[5, 0, ::2] = torch.where(listed[5, 0, ::2], z[5, 0, ::2], -torch.inf)
    # the teacher's mass all on its list (its float32 log Z leaves a rounding): no tail
    lz[6] = torch.logsumexp(val[6].double(), -1).float()
    z[6] = torch.where(listed[6], z[6], -torch.inf)
    for x in (lz, None):
        for kind in ("forward", "ce"):
            got, ref = run_distill(z, ids, val, x, kind=kind)
            assert np.isposinf(ref["per_step"][[0, 3], 0]).all() and np.isfinite(ref["per_step"][[4, 5, 6], 0]).all()
            assert np.isfinite(ref["grad"]).all()
            g = got[2]
            assert (g[5, 0][torch.isinf(z[5, 0])] == 0).all()
    # all of the student's mass on the list, the rest e^-100 to e^-400 below it
    for depth in (100.0, 400.0):
        z = logit_rows((2, 1, V), ty, 35)
        ids, val, lz = lists(2, 1, V, M, 36)
        z = (z.float() - depth).scatter(2, ids.long(), val).to(ty)
        for kind in ("forward", "ce"):
            _, ref = run_distill(z, ids, val, lz, kind=kind)
            assert np.isfinite(ref["per_step"]).all()
    # the whole vocabulary listed
    z = logit_rows((2, 1, 200), ty, 33)
    ids, val, lz = lists(2, 1, 200, 256, 34)
    for x in (lz, None):
        run_distill(z, ids, val, x)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("N,K,V,M", [
    (1, 1, 9001, 64), (70, 8, 3, 3), (64, 4, 4, 2), (300, 2, 4096, 256), (1100, 1, 38911, 64), (100, 3, 151936, 256),
    # from 160 MB of logits on, half of that in float32: rows held in registers, by their length
    (3000, 3, 10243, 20), (2700, 3, 10239, 20), (1500, 3, 19456, 64), (1400, 3, 19459, 17), (700, 3, 38912, 64),
    (2100, 1, 38913, 256), (260, 4, 77824, 64),
    # from 240 MB on, longer ones too
    (800, 2, 77825, 64), (320, 5, 77830, 130), (270, 3, 151935, 33), (401, 2, 155648, 64), (160, 5, 155649, 64)])
def test_distill_many_rows(N, K, V, M, dtype, tail):
    """Calls of few and of many rows, each side of the sizes where the gradient
    changes its launches, with empty lists, data errors and repeated ids among
    them: sampled positions against the oracle, the loss against its own steps."""
    ty = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(N * K + V)
    t = torch.randn((N, K, V), device="cuda", generator=g) * 3.0
    v, i = torch.topk(t, min(M, V), dim=-1)
    ids, val = i.to(torch.int32), v.clone()
    lz = torch.logsumexp(t / 1.5, -1)
    z = (t + torch.randn((N, K, V), device="cuda", generator=g)).to(ty)
    del t, v, i
    pos = sorted({0, 1, 2, 3, N // 3, N // 2, N - 2, N - 1} & set(range(N)))
    if N > 8:
        ids[1] = -1
        ids[2, :, 1:] = ids[2, :, :1]
        val[2, :, 1:] -= 2.0
        z[3, 0, V // 2] = torch.nan
        ids[N // 3, 0, 0] = V
        ids[N // 2, :, ::2] = -1
        z[N // 2, K - 1, :V // 2] = -torch.inf
    for gd in ({torch.float32, ty}):
        loss, per, grad = binding.distill_loss_fwd_bwd(z, ids, val, lz if tail else None, temperature=1.5, scale=0.5,
                                                       grad_dtype=gd)
        fl, fp, _ = binding.distill_loss_fwd_bwd(z, ids, val, lz if tail else None, temperature=1.5, scale=0.5,
                                                 want_grad=False)
        at = torch.tensor(pos, device="cuda")
        sub = (z[at], ids[at], val[at], lz[at] if tail else None)
        check_distill((None, per[at], grad[at]), *sub, 1.5, "forward", 0.5)
        check_distill((None, fp[at], None), *sub, 1.5, "forward", 0.5)
        for l, p in ((loss, per), (fl, fp)):
            total = 0.5 * p.double().mean(-1).sum()
            assert torch.isnan(l).all() == torch.isnan(total)
            if N <= 8:  # (the data errors make the others NaN)
                assert abs(float(l) - float(total)) <= 2.0 ** -23 * (abs(float(total)) + float(p.abs().sum()))
        # every row's gradient sums to (W + r) - W - r = 0, to within the errors of the
        # oracle's count: with a mean |d| / T of at most 15, 2 * 15 + 6 + 33 + 2 * 15 for
        # all of q, as much for the unlisted, 3 for p; and one rounding of sum |g| <= 2
        s = grad.double().sum(-1).abs()
        ok = ~torch.isnan(per)
        assert (s[ok] <= 0.5 / (K * 1.5) * (201 * 2.0 ** -24 + 2 * (2.0 ** -24 if gd == torch.float32 else 2.0 ** -8))).all()


@pytest.mark.parametrize("dtype", DT)
def test_distill_strides(dtype):
    """Slices: the first K of K + 1 steps of the lists, padded offset logits, a
    draft row shared by all steps."""
    N, K, V, M = 4, 3, 7001, 30
    big = logit_rows((N, K + 2, V + 9), TYPES[dtype], 41)
    z = big[:, 1:K + 1, 5:V + 5]
    ids, val, lz = lists(N, K + 1, V, M + 2, 42)
    i, v, l = ids[:, :K, 1:M + 1], val[:, :K, 1:M + 1], lz[:, :K]
    run_distill(z, i, v, l)
    shared = big[:, :1, :V].expand(N, K, V)
    run_distill(shared, i, v, l)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("rows", [3, 800])
def test_distill_gradient_beyond_float32(rows, tail):
    """At a temperature whose inverse float32 does not hold, tokens without mass have a gradient of 0, not NaN."""
    V = 152000
    z = -logit_rows((rows, 1, V), torch.bfloat16, 15).abs() - 1.0
    z[:, 0, 5] = 0.0
    ids = torch.tensor([5, 7], dtype=torch.int32, device="cuda").expand(rows, 1, 2).contiguous()
    val = torch.zeros(rows, 1, 2, device="cuda")
    lz = torch.full((rows, 1), 1.0, device="cuda") if tail else None
    _, _, grad = binding.distill_loss_fwd_bwd(z, ids, val, lz, temperature=1e-40, kind="ce")
    assert not torch.isnan(grad).any()
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[[5, 7]] = False
    if not tail:
        assert (grad[..., rest] == 0).all()
    assert (grad[:, 0, 5] > 0).all() and (grad[:, 0, 7] < 0).all()


def test_distill_gradient_against_differences():
    """The gradient against central differences of the float64 loss; the first log
    Z is one of another temperature, whose probabilities sum to far more than 1."""
    from oracle.rollout import distill_ref
    ids, val, lz = lists(2, 2, 50, 8, 51)
    z = logit_rows((2, 2, 50), torch.float32, 52)
    for x in (lz, torch.logsumexp(val.double() / 0.5, -1).float() + 0.1, None):
        g = binding.distill_loss_fwd_bwd(z, ids, val, x, temperature=0.5, scale=2.0)[2].double().cpu().numpy()
        zd = z.double().cpu().numpy()
        h = 1e-5

        def loss(a):
            return distill_ref(a, ids.cpu().numpy(), val.cpu().numpy(), None if x is None else x.cpu().numpy(), 0.5,
                               "forward", 2.0)

        ref = loss(zd)
        for n, k, v in [(0, 0, 0), (0, 1, 7), (1, 0, int(ids[1, 0, 0])), (1, 1, int(ids[1, 1, 7])), (1, 1, 49)]:
            a, b = zd.copy(), zd.copy()
            a[n, k, v] += h
            b[n, k, v] -= h
            # differences: h^2 / 6 times the third derivative, which is at most 2 / T^2 of the
            # gradient's unit f (W + r); the loss's own rounding (some 2^-51 of it) / h
            lim = 2 * h * h * ref["grad_unit"][n, k] + 2.0 ** -51 * abs(ref["loss"]) / h
            lim += 2.0 ** -24 * (ref["grad_err"][n, k, v] + abs(g[n, k, v]))
            assert abs((loss(a)["loss"] - loss(b)["loss"]) / (2 * h) - g[n, k, v]) <= lim


# ---- verification from probabilities ----------------------------------------------------

@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (3, 0, 9), (2, 2, 7), (5, 3, 4095), (5, 3, 4096), (4, 8, 4097),
                                   (6, 2, 8193), (7, 3, 40001), (2, 3, 151936), (300, 2, 1000)])
def test_probs_sizes(B, K, V, dtype, draft):
    p, q, ids, u, us = probs(B, K, V, TYPES[dtype], B + V, draft=draft)
    check_probs(binding.verify_probs(p, q, ids, u, us), p, q, ids, u, us)
    check_probs(binding.verify_probs(p, q, ids, u, us, want_overlap=False), p, q, ids, u, us)


@pytest.mark.parametrize("B,K,V,dtype,draft", [(13000, 3, 100, "f32", True), (12500, 3, 60, "bf16", False),
                                               (50000, 1, 20, "bf16", True), (12288, 3, 33, "f32", True),
                                               (12289, 3, 33, "f32", True)])
def test_probs_many_rows(B, K, V, dtype, draft):
    """Each side of the size from which the accept tests take their own launch."""
    p, q, ids, u, us = probs(B, K, V, TYPES[dtype], B + V, draft=draft)
    lens = (torch.arange(B, device="cuda") * 7 % (K + 1)).to(torch.int32)
    lens[5] = K + 1
    check_probs(binding.verify_probs(p, q, ids, u, us, draft_lens=lens), p, q, ids, u, us, lens)
    check_probs(binding.verify_probs(p, q, ids, u, us, want_overlap=False), p, q, ids, u, us)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("B,K,V", [(3, 2, 2047), (3, 2, 2048), (2, 2, 2049), (2, 1, 4095), (2, 1, 4096), (2, 1, 4097),
                                   (4096, 3, 33), (4097, 3, 33), (1400, 3, 4999)])
def test_probs_sub_chunks(B, K, V, dtype):
    """Each side of the sub-chunks' ends, and of the number of them where bfloat16's grow."""
    p, q, ids, u, us = probs(B, K, V, TYPES[dtype], 3 * B + V)
    for ov in (True, False):
        check_probs(binding.verify_probs(p, q, ids, u, us, want_overlap=ov), p, q, ids, u, us)


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", DT)
def test_probs_ragged(dtype, draft):
    """Rows of every length: ids, uniforms and rows behind it are not looked at."""
    B, K, V = 40, 4, 5003
    p, q, ids, u, us = probs(B, K, V, TYPES[dtype], 61, draft=draft)
    lens = (torch.arange(B, device="cuda") % (K + 1)).to(torch.int32)
    off = torch.arange(K, device="cuda")[None] >= lens[:, None]
    ids[off] = -5
    u[off] = torch.nan
    p[:, 1:][off] = torch.nan
    if q is not None:
        q[off] = torch.nan
    # the bonus row of a row is the one behind its last draft
    p[torch.arange(B, device="cuda"), lens.long()] = probs(B, 0, V, TYPES[dtype], 62)[0][:, 0]
    out = binding.verify_probs(p, q, ids, u, us, draft_lens=lens)
    ref = check_probs(out, p, q, ids, u, us, lens)
    assert (ref["accept_len"] >= 0).all()


@pytest.mark.parametrize("dtype", DT)
def test_probs_truncated_distributions(dtype):
    """Distributions with most of the vocabulary at 0, drafts outside the target's
    support, rows that do not sum to 1, a draft equal to its target."""
    ty = TYPES[dtype]
    B, K, V = 24, 3, 20001
    p, q, ids, u, us = probs(B, K, V, ty, 71)
    keep = torch.rand((B, K + 1, V), generator=torch.Generator().manual_seed(72)).cuda() < 0.001
    p = torch.where(keep, p * 300, torch.zeros_like(p))
    q[::2] = torch.where(keep[::2, :K], q[::2] * 300, torch.zeros_like(q[::2]))
    q[0] = p[0, :K]
    ids[::2] = q[::2].argmax(-1).to(torch.int32)
    check_probs(binding.verify_probs(p, q, ids, u, us), p, q, ids, u, us)
    check_probs(binding.verify_probs(p, None, ids, u, us), p, None, ids, u, us)


def test_probs_edges():
    """Uniforms of 0 and 1, comparisons that are equal, a rejected token after
    which no residual is left (the token then comes from p), single-token rows."""
    V = 6000
    p = torch.zeros((6, 2, V), device="cuda")
    q = torch.zeros((6, 1, V), device="cuda")
    p[:, :, 5] = 0.25
    p[:, :, 5000] = 0.75
    q[:, 0, 5] = 0.5
    q[:, 0, 5000] = 0.5
    ids = torch.full((6, 1), 5, dtype=torch.int32, device="cuda")
    u = torch.tensor([0.0, 0.5, 0.4999999, 1.0, 0.9, 0.9], device="cuda")[:, None].contiguous()
    us = torch.tensor([0.0, 0.3, 1.0, 0.999, 1.0, 0.2], device="cuda")
    q[4, 0] = 2 * p[4, 0]           # q covers p: the residual is empty
    q[5, 0, 5] = 0.0                # a draft token of no draft probability
    out = binding.verify_probs(p, q, ids, u, us)
    # 0.5 * 0.5 = 0.25 is not below 0.25: rejected
    assert out["accept_len"].tolist() == [1, 0, 1, 0, 0, 1]
    assert out["emitted"].tolist() == [[5, 5], [5000, -1], [5, 5000], [5000, -1], [5000, -1], [5, 5]]
    none = binding.verify_probs(p, None, ids, u, us)
    assert none["accept_len"].tolist() == [1, 0, 0, 0, 0, 0]
    assert none["emitted"][:, 0].tolist() == [5, 5000, 5000, 5000, 5000, 5000]


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("dtype", DT)
def test_probs_data_errors(dtype, draft):
    B, K, V = 14, 2, 5000
    p, q, ids, u, us = probs(B, K, V, TYPES[dtype], 81, draft=draft)
    lens = torch.full((B,), K, dtype=torch.int32, device="cuda")
    u[:] = 0.0                      # every draft passes where nothing is wrong
    ids[0, 1] = V
    ids[1, 0] = -1
    u[2, 1] = torch.nan
    u[3, 0] = -0.1
    u[4, 0] = 1.5
    us[5] = torch.nan
    us[6] = 1.5
    lens[7] = -1
    lens[8] = K + 1
    p[9, K, 77] = torch.nan         # the emitting row
    p[10, K, 78] = -1e-3
    p[11, K, 79] = torch.inf
    p[12, K] = 0.0                  # no mass
    p[13, 0, 4321] = torch.nan      # another step's row: only its overlap
    x = ids[13, 0]
    assert int(x) != 4321
    for ov in (True, False):
        out = binding.verify_probs(p, q, ids, u, us, draft_lens=lens, want_overlap=ov)
        ref = check_probs(out, p, q, ids, u, us, lens)
        assert (ref["accept_len"][:13] == -1).all() and ref["accept_len"][13] == K


@pytest.mark.parametrize("dtype", DT)
def test_probs_strides(dtype):
    big, qb, ids, u, us = probs(6, 4, 5009, TYPES[dtype], 91)
    p, q = big[:, 1:4, 3:5004], qb[:, 1:3, 3:5004]
    i = torch.clamp(ids[:, 1:3] - 3, 0, 5000).contiguous()
    check_probs(binding.verify_probs(p, q, i, u[:, :2].contiguous(), us), p, q, i, u[:, :2], us)
    one = p[:1].expand(6, 3, 5001)
    check_probs(binding.verify_probs(one, q, i, u[:, :2].contiguous(), us), one, q, i, u[:, :2], us)


# ---- together, streams, graphs -----------------------------------------------------------

def test_a_rollout_step_and_its_training_step():
    """Verify the drafts of a batch, record the target's top logits at the
    temperature of training, distil the draft from the record: with the whole
    vocabulary listed that is the forward KL of the rows themselves."""
    B, K, V, M = 6, 3, 200, 200
    tgt = logit_rows((B, K + 1, V), torch.float32, 101)
    drf = logit_rows((B, K, V), torch.float32, 102)
    p, q = torch.softmax(tgt, -1), torch.softmax(drf, -1)
    g = torch.Generator().manual_seed(103)
    ids = torch.randint(0, V, (B, K), generator=g, dtype=torch.int32).cuda()
    u, us = torch.rand((B, K), generator=g).cuda(), torch.rand(B, generator=g).cuda()
    out = binding.verify_probs(p, q, ids, u, us)
    check_probs(out, p, q, ids, u, us)
    rec = binding.top_logits(tgt, M)
    check_top(rec, tgt, M, 1.0)
    args = (rec["ids"][:, :K], rec["values"][:, :K], rec["logz"][:, :K])
    loss, per, grad = binding.distill_loss_fwd_bwd(drf, *args)
    check_distill((loss, per, grad), drf, *args, 1.0, "forward")
    kl, kps, kg = binding.kl_loss_fwd_bwd(tgt[:, :K], drf, 1.0, "forward")
    # both within their float32 sums of the same values
    assert torch.allclose(per, kps, rtol=1e-5, atol=1e-5)
    assert torch.allclose(grad, kg, rtol=1e-4, atol=1e-7)


def test_two_rollout_threads():
    """Calls from two host threads at once, each on its own stream."""
    import threading
    want = {s: [_bits(c()) for c in _calls(s)] for s in (181, 191)}
    torch.cuda.synchronize()
    errors = []

    def work(seed):
        try:
            calls = _calls(seed)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for _ in range(5):
                    for w, c in zip(want[seed], calls):
                        assert all(torch.equal(x, y) for x, y in zip(w, _bits(c())))
            s.synchronize()
        except BaseException as e:  # noqa: BLE001 (handed to the test's thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(s,)) for s in want]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def _calls(seed):
    z = logit_rows((5, 2, 30011), torch.bfloat16, seed)
    ids, val, lz = lists(5, 2, 30011, 32, seed + 1)
    p, q, di, u, us = probs(9, 2, 30011, torch.float32, seed + 2)
    return [lambda: tuple(binding.top_logits(z, 48).values()),
            lambda: binding.distill_loss_fwd_bwd(z, ids, val, lz),
            lambda: tuple(binding.verify_probs(p, q, di, u, us).values())]


def _bits(ts):
    return [t.clone().view(torch.uint8) for t in ts]


def test_repeated_calls_give_the_same_bits():
    for call in _calls(111):
        a = _bits(call())
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(a, _bits(call())))


def test_streams():
    """Calls on two streams at once, each with its own scratch memory."""
    calls = _calls(121)
    want = [_bits(c()) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for rep in range(4):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append([c() for c in calls])
    torch.cuda.synchronize()
    for outs in got:
        for w, o in zip(want, outs):
            assert all(torch.equal(x, y) for x, y in zip(w, _bits(o)))


def test_captured_graphs():
    """Two graphs captured one after another and replayed several times, eager
    calls of another size between the replays."""
    graphs = []
    for seed in (131, 141):
        calls = _calls(seed)
        want = [_bits(c()) for c in calls]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = [c() for c in calls]
        graphs.append((g, outs, want, calls))
    other = _calls(151)
    for rep in range(4):
        for g, outs, want, _ in graphs:
            for o in outs:
                for t in o:
                    t.zero_()
            g.replay()
            torch.cuda.synchronize()
            for w, o in zip(want, outs):
                assert all(torch.equal(x, y) for x, y in zip(w, _bits(o)))
            for c in other:
                c()
            torch.cuda.synchronize()


def test_captured_calls_of_many_rows():
    """The launches of large calls (rows handed out by a counter, split rows merged,
    accept tests in a launch of their own), captured together and replayed: each
    replay has the eager calls' bits, also after eager calls in between, and
    nothing is written beside the gradient."""
    N, K, V, M = 900, 3, 32003, 40  # 173 MB of bfloat16 logits
    z = logit_rows((N, K, V), torch.bfloat16, 201)
    ids, val, lz = lists(N, K, V, M, 202)
    ids[5] = -1
    z[7, 1, 3] = torch.nan
    p, q, di, u, us = probs(20000, 2, 24, torch.bfloat16, 203)
    buf = torch.full((N * K * V + 64,), 3.0, device="cuda", dtype=torch.bfloat16)
    g = buf[31:31 + N * K * V].view(N, K, V)

    def step():
        return (tuple(binding.top_logits(z[:4], M).values())
                + binding.distill_loss_fwd_bwd(z, ids, val, lz, scale=0.5, grad_out=g)[:2] + (g,)
                + tuple(binding.verify_probs(p, q, di, u, us).values()))

    want = _bits(step())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for rep in range(4):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(w, o) for w, o in zip(want, _bits(outs)))
        assert (buf[:31] == 3.0).all() and (buf[-33:] == 3.0).all()
        binding.distill_loss_fwd_bwd(z[:850], ids[:850], val[:850], lz[:850])
        torch.cuda.synchronize()


def test_offsets_beyond_32_bits():
    """Rows that start 2^31 elements and more behind the first, and a gradient of more elements than that."""
    V, far = 9001, 2 ** 31 + 12
    buf = torch.empty(far + 4 * V, device="cuda")

    def spread(t):  # the same values, the second entry of the first dimension far away
        o = buf.as_strided(t.shape, (far, V, 1))
        o.copy_(t)
        return o

    z = logit_rows((2, 3, V), torch.float32, 211)
    check_top(binding.top_logits(spread(z), 30), z, 30, 1.0)
    ids, val, lz = lists(2, 3, V, 30, 212)
    check_distill(binding.distill_loss_fwd_bwd(spread(z), ids, val, lz), z, ids, val, lz, 1.0, "forward")
    p, q, di, u, us = probs(2, 2, V, torch.float32, 213)
    check_probs(binding.verify_probs(spread(p), q, di, u, us), p, q, di, u, us)
    check_probs(binding.verify_probs(p, spread(q), di, u, us), p, q, di, u, us)
    del buf
    N, V, M = 14200, 151936, 16
    row = logit_rows((1, 1, V), torch.bfloat16, 214).expand(N, 1, V)
    ids, val, lz = (t.expand(N, *t.shape[1:]) for t in lists(1, 1, V, M, 215))
    _, per, g = binding.distill_loss_fwd_bwd(row, ids, val, lz, grad_dtype=torch.bfloat16)
    assert g.numel() > 2 ** 31
    check_distill((None, per[-1:], g[-1:]), row[-1:], ids[-1:], val[-1:], lz[-1:], 1.0, "forward")
    assert (per == per[-1]).all()
    for n in (0, N // 2, N - 2):
        assert torch.equal(g[n], g[-1])


def test_given_outputs_and_workspace():
    z = logit_rows((4, 9001), torch.float32, 161)
    ws = torch.empty(binding.top_logits_workspace_size(4, 1, 9001, 20, torch.float32), dtype=torch.uint8, device="cuda")
    out = {"ids": torch.empty((4, 20), dtype=torch.int32, device="cuda"), "values": torch.empty((4, 20), device="cuda")}
    got = binding.top_logits(z, 20, ws=ws, out=out)
    assert got is out
    check_top(out, z, 20, 1.0, want_logz=False)
    ids, val, lz = lists(4, 1, 9001, 12, 162)
    g = torch.full((4, 1, 9001), 7.0, device="cuda")
    zz = z.view(4, 1, 9001)
    got = binding.distill_loss_fwd_bwd(zz, ids, val, lz, grad_out=g, want_per_step=False)
    assert got[1] is None and got[2] is g
    check_distill(got, zz, ids, val, lz, 1.0, "forward")
    with pytest.raises(ValueError):
        binding.distill_loss_fwd_bwd(zz, ids, val, lz, grad_out=zz)
    with pytest.raises(binding.SpecError):
        binding.top_logits(z, 20, ws=ws[:256])


@pytest.mark.parametrize("dtype", DT)
def test_guard_bytes(dtype):
    """Nothing is written outside the outputs."""
    N, K, V, M = 3, 2, 4099, 11
    z = logit_rows((N, K, V), TYPES[dtype], 171)
    ids, val, lz = lists(N, K, V, M, 172)
    buf = torch.full((N * K * V + 64,), 3.0, device="cuda", dtype=TYPES[dtype])
    g = buf[32:32 + N * K * V].view(N, K, V)
    binding.distill_loss_fwd_bwd(z, ids, val, lz, grad_out=g)
    assert (buf[:32] == 3.0).all() and (buf[-32:] == 3.0).all()
    ib = torch.full((N * K * M + 64,), 77, device="cuda", dtype=torch.int32)
    vb = torch.full((N * K * M + 64,), 7.0, device="cuda")
    binding.top_logits(z, M, out={"ids": ib[32:-32].view(N, K, M), "values": vb[32:-32].view(N, K, M)})
    assert (ib[:32] == 77).all() and (ib[-32:] == 77).all() and (vb[:32] == 7.0).all() and (vb[-32:] == 7.0).all()
