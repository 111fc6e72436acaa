"""Operators of token policies (paper_2104_06272_amd/tokens.py) against a plain 64-bit statement of the same formulas.

Tolerances count roundings (u = 2^-24 is half a step of binary32).  A sum of V exponentials is off by at most
(chain + 2 |t|) u of itself, where a chain of additions is no longer than V / 64 + 64 (elements a lane adds, and the joins)
and the exponent t = log2 of an element's share is rounded a few times; outputs in fp32 add u, in bf16 2^-9 and in fp16
2^-12 of the value (half a step is eps / 2 of the value at most), and what lies under the smallest normal number may be lost."""
import ctypes as C
import math
import os
import sys

import numpy as np
import pytest
import torch

from paper_2104_06272_amd import binding, tokens

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
gpu = pytest.mark.gpu


def roundings(V):
    return (V / 64 + 64) * U


# ---- the plain statement, float64 on the CPU -----------------------------------------------------------------------
def ref_rows(logits, target, scale):
    """log p, log-probability of the target, log-sum-exp, entropy, rows that take part"""
    z = logits.detach().cpu().double() * scale
    t = target.cpu().to(torch.int64)
    N, V = z.shape
    on = (t >= 0) & (t < V)
    z = torch.where(on[:, None], z, torch.zeros_like(z))
    m = z.max(1).values
    empty = torch.isneginf(m)
    shifted = z - torch.where(empty, 0.0, m)[:, None]             # (64 bits, too, lose log V beside the lowest value of a type)
    log_s = torch.log(torch.exp(shifted).sum(1))
    logs, lse = shifted - log_s[:, None], m + log_s
    p = torch.exp(logs)
    logs[empty] = -math.inf
    p[empty] = 0.0
    H = -torch.where(p > 0, p * logs, torch.where(torch.isnan(p), p, torch.zeros_like(p))).sum(1)
    lp = logs.gather(1, t.clamp(0, V - 1)[:, None]).reshape(-1)
    zero = torch.zeros_like(lp)
    return dict(logs=logs, p=p, lp=torch.where(on, lp, zero), lse=torch.where(on, lse, zero), H=torch.where(on, H, zero), on=on, t=t, empty=empty)


def ref_gradient(x, g, e, scale):
    """scale (g ([j = a] - p_j) - e p_j (log p_j + H)), and the sum of the terms' sizes, which roundings are measured on"""
    p, logs = x["p"], torch.where(x["p"] > 0, x["logs"], torch.zeros_like(x["logs"]))
    g, e = torch.where(x["on"] & ~x["empty"], g, 0.0)[:, None], torch.where(x["on"] & ~x["empty"], e, 0.0)[:, None]
    hot = torch.zeros_like(p)
    hot[torch.arange(len(p)), x["t"].clamp(0, p.shape[1] - 1)] = 1.0
    H = x["H"][:, None]
    d = scale * (g * (hot - p) - e * p * (logs + H))
    size = scale * (g.abs() * (hot + p * (1 + logs.abs())) + e.abs() * p * (logs.abs() + H.abs() + 1) * (1 + logs.abs()))
    return torch.where(x["on"][:, None], d, 0.0), torch.where(x["on"][:, None], size, 0.0)


def ref_policy(x, old, adv, low, high, kl_coef, ref, ent, weight, norm):
    on, lp = x["on"].clone(), x["lp"]
    w = torch.ones_like(lp) if weight is None else weight.cpu().double()
    on &= w != 0
    w = torch.where(on, w, 0.0)
    W = norm or float(w.sum())
    A = adv.cpu().double()
    r = torch.exp(lp - old.cpu().double())
    plain, clip = r * A, r.clamp(1 - low, 1 + high) * A
    inside = plain <= clip
    count = on & ~x["empty"]
    d = torch.zeros_like(lp) if ref is None else ref.cpu().double() - lp
    kl = torch.exp(d) - d - 1
    g = torch.where(inside, -plain, 0.0) + kl_coef * (1 - torch.exp(d))
    inv = 1.0 / W if W else 0.0
    zero = torch.zeros_like(lp)
    take = lambda v: float((w * torch.where(count, v, zero)).sum()) * inv
    policy, k, H = take(-torch.minimum(plain, clip)), take(kl), take(x["H"])
    stats = [policy + kl_coef * k - ent * H, policy, k, H, take((~inside).double()), take(r), W, float(on.sum())]
    # g is a sum of two terms, each of which an error of lp changes by its own size (d(r A) = r A dlp, d(k e^d) = -k e^d dlp)
    g_size = torch.where(inside, plain.abs(), 0.0) + kl_coef * (1 + torch.exp(d))
    return stats, torch.where(count, g * w * inv, zero), torch.where(count, -ent * w * inv, zero), on, torch.where(count, g_size * w * inv, zero)


def rows_of(layout, count, length, lengths):
    out, at = [], 0
    for s in range(count):
        n = lengths[s]
        if layout == "packed":
            out.append(np.arange(at, at + n)); at += n
        elif layout == "batch":
            out.append(s * length + np.arange(n))
        else:
            out.append(np.arange(n) * count + s)
    return out


def ref_preference(x, rows, beta, margin, mean, ref, label, weight, norm):
    P = len(rows) // 2
    lp = x["lp"] - (0.0 if ref is None else ref.cpu().double())
    D, n = np.zeros(2 * P), np.zeros(2 * P)
    for s, r in enumerate(rows):
        r = r[x["on"].numpy()[r]]
        n[s] = len(r)
        D[s] = float(lp[r].sum()) / (max(1, len(r)) if mean else 1)
    h = beta * (D[:P] - D[P:]) - margin
    y = np.ones(P) if label is None else label.cpu().double().numpy()
    w = np.ones(P) if weight is None else weight.cpu().double().numpy()
    W = norm or w.sum()
    inv = 1.0 / W if W else 0.0
    up, down = np.logaddexp(0.0, -h), np.logaddexp(0.0, h)
    loss = np.where(y != 0, y * up, 0.0) + np.where(y != 1, (1 - y) * down, 0.0)
    dh = ((1 - y) / (1 + np.exp(-h)) - y / (1 + np.exp(h))) * w * inv * beta
    g = torch.zeros(len(x["lp"]), dtype=torch.float64)
    for s, r in enumerate(rows):
        g[r] = (dh[s] if s < P else -dh[s - P]) / (max(1.0, n[s]) if mean else 1.0)
    on = w != 0
    with np.errstate(invalid="ignore"):
        t = lambda v: float((w * v)[on].sum()) * inv
        stats = [t(loss), t(h > 0), beta * t(D[:P]), beta * t(D[P:]), t(h), W, float(on.sum()), float((n[:P] + n[P:])[on].sum())]
    return stats, h, g, n


def ref_returns(reward, value, rows, gamma, lam, done, bootstrap):
    r, v = reward.cpu().double().numpy(), value.cpu().double().numpy()
    d = np.zeros(len(r)) if done is None else done.cpu().numpy() != 0
    adv, ret = np.zeros(len(r)), np.zeros(len(r))
    for s, idx in enumerate(rows):
        G = V = 0.0 if bootstrap is None else float(bootstrap[s])
        for i in idx[::-1]:
            G = r[i] + (0.0 if d[i] else gamma) * ((1 - lam) * V + lam * G)
            V = v[i]
            ret[i], adv[i] = G, G - V
    return adv, ret


# ---- comparisons -----------------------------------------------------------------------------------------------------
def close(got, want, tol, what):
    got, want = got.detach().cpu().double(), torch.as_tensor(want).double()
    assert got.shape == want.shape, what
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~same & ~((got - want).abs() <= torch.as_tensor(tol))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {torch.nonzero(bad)[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


def close_logp(r, x, V):
    close(r.logp, x["lp"], U * x["lp"].abs().nan_to_num(0, 0, 0) + 2 * roundings(V), "logp")
    close(r.lse, x["lse"], U * x["lse"].abs().nan_to_num(0, 0, 0) + 2 * roundings(V), "lse")


def close_gradient(got, want, size, V, dtype):
    fi = torch.finfo(dtype)
    tiny = fi.smallest_normal * (1.0 if dtype == torch.float32 else fi.eps)           # flushed exponentials; subnormals' half steps
    size = size.nan_to_num(0, 0, 0)
    want = torch.where(torch.isinf(want.to(dtype)), torch.sign(want) * math.inf, want)   # what the type cannot hold rounds to infinity
    close(got, want, fi.eps / 2 * want.abs().nan_to_num(0, 0, 0) + 4 * roundings(V) * size + tiny, "gradient")


def make_logits(N, V, dtype, pad=0, seed=0, device="cuda", std=2.5):
    g = torch.Generator().manual_seed(1000 * seed + N * 7 + V)
    z = torch.randn(N, V, generator=g) * std
    room = torch.full((N, V + pad), 7.0, dtype=DT[dtype], device=device)
    room[:, :V] = z.to(DT[dtype]).to(device)
    return room[:, :V], room, g


def make_target(N, V, g, kind=torch.int64, skip=0.0, device="cuda"):
    t = torch.randint(0, V, (N,), generator=g)
    if skip:
        t[torch.rand(N, generator=g) < skip] = -1
    return t.to(kind).to(device)


SIZES = [(1, 1, 0), (3, 2, 0), (70, 3, 1), (5, 7, 0), (33, 8, 2), (9, 63, 1), (4, 64, 0), (130, 65, 0), (7, 255, 3), (3, 256, 0), (6, 1000, 0),
         (5, 1024, 0), (4, 1025, 7), (3, 2049, 0), (2, 4099, 1), (3, 8192, 8), (2, 16411, 0), (3, 32768, 0), (2, 50001, 3), (1, 65537, 0),
         (2, 131072, 0), (1, 200003, 0), (1, 262145, 0),
         # every form of short and long rows, and as many rows as take more than one workgroup's sums
         (40, 100, 0), (40, 128, 2), (33, 300, 1), (20, 511, 0), (20, 513, 0), (9, 1023, 1), (5, 1500, 1), (4, 3000, 0), (3, 12000, 1), (2, 40000, 0), (2, 100003, 5),
         (2500, 5, 0), (3000, 600, 1), (700, 2100, 1), (5000, 40, 3)]


# ---- CPU: the statement itself, and refusals -------------------------------------------------------------------------
def test_reference_gradients_are_differences():
    z, _, g = make_logits(4, 6, "fp32", device="cpu")
    z = z.double()
    t = torch.tensor([0, 5, -1, 2])
    old, adv, ref = torch.randn(3, 4, generator=g).double()
    old -= 2.0; ref -= 2.0
    w = torch.tensor([1.0, 0.5, 1.0, 2.0])

    def policy(z):
        return ref_policy(ref_rows(z, t, 0.7), old, adv, 0.2, 0.3, 0.1, ref, 0.05, w, 0.0)
    rows = rows_of("packed", 4, 0, [1, 1, 1, 1])
    rows = [np.array([0, 1]), np.array([2]), np.array([3]), np.array([], int)]
    label, pw = torch.tensor([0.8, 0.1]), torch.tensor([1.0, 3.0])

    def preference(z):
        return ref_preference(ref_rows(z, t, 0.7), rows, 0.6, 0.2, True, ref, label, pw, 0.0)
    x = ref_rows(z, t, 0.7)
    _, g1, g2, _, _ = policy(z)
    by_formula = ref_gradient(x, g1, g2, 0.7)[0], ref_gradient(x, preference(z)[2], torch.zeros(4).double(), 0.7)[0]
    step = 1e-5
    for f, want in zip((policy, preference), by_formula):
        for i in range(4):
            for j in range(6):
                d = torch.zeros_like(z); d[i, j] = step
                diff = (f(z + d)[0][0] - f(z - d)[0][0]) / (2 * step)
                assert abs(diff - float(want[i, j])) < 1e-8, (i, j)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2104_06272_amd import build
        build.build(verbose=False)
    return binding.load()


FAKE = 0x10000000                                                 # never dereferenced: every call below is refused on the host


def _rows(**over):
    x = dict(logits=FAKE, rows=8, vocab=100, row_stride=100, target=FAKE + 0x100000, type=1, target_type=2, scale=1.0)
    x.update(over)
    return binding.Rows(*[x[k] for k, _ in binding.Rows._fields_])


def _policy(**over):
    a = dict(logp_old=FAKE, adv=FAKE, logp_ref=None, weight=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, norm=0.0, grad_scale=1.0,
             stats=FAKE, logp=None, dlogits=FAKE + 0x200000, grad_stride=100)
    a.update(over)
    return binding.PolicyArgs(*[a[k] for k, _ in binding.PolicyArgs._fields_])


BAD_ROWS = [dict(type=3), dict(type=-1), dict(target_type=3), dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=1 << 28), dict(row_stride=99), dict(scale=0.0),
            dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-7), dict(logits=None), dict(target=None), dict(row_stride=1 << 50), dict(rows=(1 << 31) - 1, row_stride=1 << 31), dict(row_stride=-100)]


@pytest.mark.parametrize("over", BAD_ROWS, ids=str)
def test_rows_are_checked_on_the_host(lib, over):
    x = _rows(**over)
    assert lib.anakin_policy_loss(x, _policy(), FAKE, 1 << 30, None) == binding.E_INVALID_ARG
    assert lib.anakin_last_error(None)
    assert lib.anakin_token_logprobs(x, FAKE, FAKE, None, None) == binding.E_INVALID_ARG
    assert lib.anakin_token_logprobs_backward(x, FAKE, None, FAKE, None, FAKE + 0x200000, 100, None) == binding.E_INVALID_ARG


@pytest.mark.parametrize("over,code", [
    (dict(stats=None), -1), (dict(logp_old=None), -1), (dict(adv=None), -1), (dict(clip_low=-0.1), -1), (dict(clip_low=1.5), -1), (dict(clip_high=-0.1), -1),
    (dict(clip_high=math.inf), -1), (dict(clip_low=math.nan), -1), (dict(kl_coef=0.1), -1), (dict(kl_coef=math.nan), -1), (dict(entropy_coef=math.inf), -1),
    (dict(grad_scale=math.nan), -1), (dict(norm=-1.0), -1), (dict(grad_stride=99), -1), (dict(dlogits=FAKE + 16), -1), (dict(dlogits=FAKE, grad_stride=101), -1),
    (dict(dlogits=FAKE + 0x200001), -4)], ids=str)
def test_policy_arguments_are_checked_on_the_host(lib, over, code):
    assert lib.anakin_policy_loss(_rows(), _policy(**over), FAKE, 1 << 30, None) == code


def test_workspaces_are_checked_on_the_host(lib):
    need = lib.anakin_rows_workspace_bytes(8, 100, 0)
    assert need > 0 and need % 256 == 0
    assert lib.anakin_policy_loss(_rows(), _policy(), FAKE, need - 1, None) == binding.E_WORKSPACE_TOO_SMALL and b"need" in lib.anakin_last_error(None)
    assert lib.anakin_policy_loss(_rows(), _policy(), FAKE + 8, need, None) == binding.E_MISALIGNED
    assert lib.anakin_policy_loss(_rows(), _policy(), None, need, None) == binding.E_INVALID_ARG
    assert lib.anakin_policy_loss(None, _policy(), FAKE, need, None) == binding.E_INVALID_ARG
    assert lib.anakin_policy_loss(_rows(), None, FAKE, need, None) == binding.E_INVALID_ARG
    for bad in ((-1, 5, 0), (5, 0, 0), (1 << 31, 5, 0), (5, 1 << 28, 0), (5, 5, -1)):
        assert lib.anakin_rows_workspace_bytes(*bad) == 0
    assert lib.anakin_returns_workspace_bytes(-1, 1) == 0 and lib.anakin_returns_workspace_bytes(1, -1) == 0
    assert lib.anakin_token_logprobs(_rows(logits=FAKE + 1), FAKE, FAKE, None, None) == binding.E_MISALIGNED
    assert lib.anakin_token_logprobs(_rows(target=FAKE + 4), FAKE, FAKE, None, None) == binding.E_MISALIGNED
    assert lib.anakin_token_logprobs(_rows(), None, FAKE, None, None) == binding.E_INVALID_ARG
    assert lib.anakin_token_logprobs_backward(_rows(), FAKE, None, FAKE, FAKE, FAKE + 0x200000, 100, None) == binding.E_INVALID_ARG
    assert lib.anakin_token_logprobs_backward(_rows(), FAKE, None, FAKE, None, None, 100, None) == binding.E_INVALID_ARG


def _seq(layout=0, count=4, length=0, offsets=FAKE, lengths=None):
    return binding.SequenceArgs(layout, count, length, offsets, lengths)


def _pref(**over):
    a = dict(logp_ref=None, label=None, weight=None, beta=0.1, margin=0.0, norm=0.0, grad_scale=1.0, mean=0, stats=FAKE, margins=None, logp=None, dlogits=None, grad_stride=0)
    a.update(over)
    return binding.PreferenceArgs(*[a[k] for k, _ in binding.PreferenceArgs._fields_])


def _ret(**over):
    a = dict(rows=8, reward=FAKE, value=FAKE, done=None, bootstrap=None, value_type=0, gamma=1.0, lambda_=0.9, adv=FAKE + 0x100000, ret=FAKE + 0x200000)
    a.update(over)
    return binding.ReturnsArgs(*[a[k] for k, _ in binding.ReturnsArgs._fields_])


@pytest.mark.parametrize("over", [dict(layout=3), dict(count=-2), dict(offsets=None), dict(layout=1, length=3), dict(layout=2, length=1 << 40), dict(layout=1, length=-2),
                                  dict(layout=2, count=1 << 30, length=1 << 30)], ids=str)
def test_sequences_are_checked_on_the_host(lib, over):
    assert lib.anakin_preference_loss(_rows(), _seq(**over), _pref(), FAKE, 1 << 30, None) == binding.E_INVALID_ARG
    assert lib.anakin_lambda_returns(_seq(**over), _ret(), FAKE, 1 << 30, None) == binding.E_INVALID_ARG


def test_pairs_and_returns_are_checked_on_the_host(lib):
    assert lib.anakin_preference_loss(_rows(), _seq(count=3), _pref(), FAKE, 1 << 30, None) == binding.E_INVALID_ARG
    assert lib.anakin_preference_loss(_rows(), None, _pref(), FAKE, 1 << 30, None) == binding.E_INVALID_ARG
    assert lib.anakin_preference_loss(_rows(), _seq(), None, FAKE, 1 << 30, None) == binding.E_INVALID_ARG
    assert lib.anakin_preference_loss(_rows(), _seq(offsets=FAKE + 4), _pref(), FAKE, 1 << 30, None) == binding.E_MISALIGNED
    assert lib.anakin_preference_loss(_rows(), _seq(), _pref(), FAKE, 256, None) == binding.E_WORKSPACE_TOO_SMALL
    for over in (dict(beta=math.nan), dict(margin=math.inf), dict(norm=-1.0), dict(stats=None), dict(dlogits=FAKE + 0x200000, grad_stride=3)):
        assert lib.anakin_preference_loss(_rows(), _seq(), _pref(**over), FAKE, 1 << 30, None) == binding.E_INVALID_ARG, over
    for over in (dict(gamma=1.5), dict(gamma=math.nan), dict(lambda_=-0.1), dict(value_type=4), dict(reward=None), dict(value=None), dict(adv=None), dict(ret=None), dict(rows=-1),
                 dict(adv=FAKE), dict(ret=FAKE + 28), dict(ret=FAKE + 0x100000), dict(done=FAKE + 0x100000), dict(bootstrap=FAKE + 0x200010)):
        assert lib.anakin_lambda_returns(_seq(), _ret(**over), FAKE, 1 << 30, None) == binding.E_INVALID_ARG, over
    assert lib.anakin_lambda_returns(_seq(), None, FAKE, 1 << 30, None) == binding.E_INVALID_ARG
    assert lib.anakin_lambda_returns(_seq(), _ret(), FAKE, 0, None) == binding.E_WORKSPACE_TOO_SMALL


def test_no_gpu_tensors_means_error_not_fallback():
    z = torch.zeros(3, 5)
    t = torch.zeros(3, dtype=torch.int64)
    f = torch.zeros(3)
    for call in (lambda: tokens.logprobs(z, t), lambda: tokens.logprobs_backward(z, t, f, f), lambda: tokens.policy_loss(z, t, f, f),
                 lambda: tokens.preference_loss(z, t, tokens.batch_major(1, 3)), lambda: tokens.lambda_returns(f, f, tokens.batch_major(1, 3))):
        with pytest.raises(RuntimeError):
            call()
    with pytest.raises(binding.AnakinError):
        tokens.packed(torch.zeros(3, dtype=torch.int32))
    with pytest.raises(binding.AnakinError):
        tokens.batch_major(3, 4, lengths=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(binding.AnakinError):
        tokens.time_major(3, 4, lengths=torch.zeros(2, dtype=torch.int32))


# ---- GPU ---------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,V,pad", SIZES)
def test_logprobs_and_their_backward_pass(dtype, N, V, pad):
    z, room, g = make_logits(N, V, dtype, pad)
    before = room.clone()
    t = make_target(N, V, g, [torch.int64, torch.int32][N % 2], skip=0.2 if N > 4 else 0.0)
    scale = [1.0, 1.25, 0.37][V % 3]
    r = tokens.logprobs(z, t, scale=scale, entropy=True)
    x = ref_rows(z, t, scale)
    close_logp(r, x, V)
    close(r.entropy, x["H"], (4 + 2 * x["H"].abs()) * roundings(V), "entropy")
    r2 = tokens.logprobs(z, t, scale=scale)
    assert torch.equal(r2.logp, r.logp) and torch.equal(r2.lse, r.lse) and r2.entropy is None
    up = 256.0 if dtype == "fp16" else 1.0
    g1, g2 = torch.randn(2, N, generator=g) * up
    for e in (None, g2):
        d = tokens.logprobs_backward(z, t, r.lse, g1.cuda(), entropy=r.entropy, grad_entropy=None if e is None else e.cuda(), scale=scale)
        want, size = ref_gradient(x, g1.double(), torch.zeros(N).double() if e is None else e.double(), scale)
        # the lse handed over is rounded to fp32 itself: u |lse| more in every exponent
        close_gradient(d, want, size * (1 + x["lse"].abs()[:, None]), V, DT[dtype])
    assert torch.equal(room, before)
    own = z.clone()
    d2 = tokens.logprobs_backward(own, t, r.lse, g1.cuda(), entropy=r.entropy, grad_entropy=g2.cuda(), scale=scale, out=own)
    assert d2 is own and torch.equal(d2, d)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,V,pad", SIZES)
def test_policy_loss(dtype, N, V, pad):
    z, room, g = make_logits(N, V, dtype, pad, seed=1)
    before = room.clone()
    t = make_target(N, V, g, torch.uint8 if V < 256 else torch.int64, skip=0.2 if N > 4 and V > 255 else 0.0)
    scale = [1.0, 0.8][V % 2]
    x = ref_rows(z, t, scale)
    # log ratios of 0.1, a quarter of them outside the clipping range, none within roundings of its borders
    shift = 0.15 * torch.randn(N, generator=g).double()
    for border in (math.log(0.8), math.log(1.28)):
        shift = torch.where((shift - border).abs() < 0.01, shift + 0.02, shift)
    old = (x["lp"] - shift).float()
    adv, ref = torch.randn(N, generator=g), (x["lp"] + 0.3 * torch.randn(N, generator=g)).float()
    weight = torch.rand(N, generator=g) * (torch.rand(N, generator=g) < 0.8)
    up = 128.0 * N if dtype == "fp16" else 1.0
    for kl, ent, w, norm in ((0.0, 0.0, None, 0.0), (0.3, 0.05, weight, 0.0), (0.0, 0.02, weight, 3.5), (0.2, 0.0, None, 0.0)):
        cu = lambda v: None if v is None else v.cuda()
        r = tokens.policy_loss(z, t, cu(old), cu(adv), clip=(0.2, 0.28), kl_coef=kl, logp_ref=cu(ref) if kl else None, entropy_coef=ent, weight=cu(w), norm=norm,
                               scale=scale, grad_scale=up)
        stats, g1, g2, on, g_size = ref_policy(x, old, adv, 0.2, 0.28, kl, ref if kl else None, ent, w, norm)
        close(r.logp, torch.where(on, x["lp"], 0.0), U * x["lp"].abs() + 2 * roundings(V), "logp")
        size = 4.0 * (1 + torch.tensor(stats, dtype=torch.float64).abs() + float(adv.abs().max())) * (1.0 if not norm else max(1.0, float(weight.sum()) / norm))
        close(r.stats, torch.tensor(stats, dtype=torch.float64), size * roundings(V), "stats")
        want, _ = ref_gradient(x, g1 * up, g2 * up, scale)
        # the ratio carries the roundings of lp: an absolute error of lp is a relative one of each term of g
        _, sz = ref_gradient(x, g_size * up, g2 * up, scale)
        close_gradient(r.dlogits, want, 3 * sz, V, DT[dtype])
        alone = tokens.policy_loss(z, t, cu(old), cu(adv), clip=(0.2, 0.28), kl_coef=kl, logp_ref=cu(ref) if kl else None, entropy_coef=ent, weight=cu(w), norm=norm,
                                   scale=scale, gradient=False)
        assert alone.dlogits is None
        close(alone.stats, torch.tensor(stats, dtype=torch.float64), size * roundings(V), "stats of the loss alone")
        close(alone.logp, torch.where(on, x["lp"], 0.0), U * x["lp"].abs() + 2 * roundings(V), "logp of the loss alone")
    assert torch.equal(room, before)
    own = room.clone()
    again = tokens.policy_loss(own[:, :V], t, old.cuda(), adv.cuda(), clip=(0.2, 0.28), kl_coef=0.2, logp_ref=ref.cuda(), scale=scale, grad_scale=up, out=own[:, :V])
    assert torch.equal(again.dlogits, r.dlogits) and torch.equal(again.stats, r.stats)
    assert torch.equal(own[:, V:], room[:, V:])


def _special(dtype, V):
    """rows of logits that want care, and targets"""
    low = float(torch.finfo(DT[dtype]).min)
    big = float(torch.finfo(DT[dtype]).max)
    g = torch.Generator().manual_seed(V)
    base = torch.randn(V, generator=g)
    rows, t = [], []

    def add(row, target):
        rows.append(row.clone()); t.append(target)
    r = base.clone(); r[1::2] = -math.inf; add(r, 0); add(r, 1)                     # half forbidden; a forbidden target
    r = base.clone(); r[1::2] = low; add(r, 0); add(r, 1)                            # masked by the lowest value
    add(torch.full((V,), -math.inf), 0)                                              # nothing allowed
    add(torch.full((V,), low), V - 1)                                                # all the lowest value: all alike
    add(torch.full((V,), big), 0)
    r = torch.full((V,), low); r[V // 2] = -math.inf; add(r, 0)
    r = torch.full((V,), -math.inf); r[V - 1] = 3.0; add(r, V - 1)                   # one choice left
    r = torch.full((V,), -math.inf); r[0] = low; add(r, 0)
    add(torch.full((V,), math.nan), -1); add(torch.full((V,), math.inf), -1)         # left out: may hold anything
    add(torch.full((V,), math.nan), V); add(base, V)
    add(base * 0.0, 0)
    add(base + 3e4 if dtype == "fp16" else base + 1e6, 2 % V)
    return torch.stack(rows).to(DT[dtype]), torch.tensor(t)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [2, 9, 64, 300, 1030, 5000, 33000, 132000])
def test_masks_and_extremes(dtype, V):
    z, t = _special(dtype, V)
    x = ref_rows(z, t, 1.0)
    zc, tc = z.cuda(), t.cuda()
    r = tokens.logprobs(zc, tc, entropy=True)
    close_logp(r, x, V)
    close(r.entropy, torch.where(x["empty"], 0.0, x["H"]), (4 + 2 * x["H"].abs()) * roundings(V), "entropy")
    N = len(t)
    g = torch.Generator().manual_seed(1)
    adv, w = torch.randn(N, generator=g), torch.rand(N, generator=g) + 0.1
    old = torch.where(torch.isfinite(x["lp"]), x["lp"] - 0.1, -2.0).float()
    p = tokens.policy_loss(zc, tc, old.cuda(), adv.cuda(), entropy_coef=0.01, weight=w.cuda(), grad_scale=64.0)
    stats, g1, g2, on, _ = ref_policy(x, old, adv, 0.2, 0.2, 0.0, None, 0.01, w, 0.0)
    want, size = ref_gradient(x, 64 * g1, 64 * g2, 1.0)
    close(p.stats, torch.tensor(stats, dtype=torch.float64), 4 * (1 + torch.tensor(stats).double().abs() + 3) * roundings(V), "stats")
    close_gradient(p.dlogits, want, 3 * size, V, DT[dtype])
    assert torch.isfinite(p.dlogits).all()
    d = tokens.logprobs_backward(zc[:4], tc[:4], r.lse[:4], adv[:4].cuda(), entropy=r.entropy[:4], grad_entropy=w[:4].cuda())
    x4 = {k: v[:4] for k, v in x.items()}
    want, size = ref_gradient(x4, adv[:4].double(), w[:4].double(), 1.0)
    close_gradient(d, want, size * (1 + x4["lse"].abs()[:, None]), V, DT[dtype])


@gpu
@pytest.mark.parametrize("V", [5, 700, 40000])
def test_a_nan_stays_in_its_row(V):
    z, _, g = make_logits(6, V, "fp32")
    z[2, V - 1] = math.nan
    z[4, 0] = math.inf
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    r = tokens.logprobs(z, t, entropy=True)
    assert torch.isnan(r.logp[[2, 4]]).all() and torch.isnan(r.lse[2]) and torch.isfinite(r.logp[[0, 1, 3, 5]]).all()
    p = tokens.policy_loss(z, t, torch.zeros(6, device="cuda"), torch.ones(6, device="cuda"))
    assert torch.isnan(p.loss) and torch.isnan(p.dlogits[2]).all() and torch.isfinite(p.dlogits[[0, 1, 3, 5]]).all()


@gpu
@pytest.mark.parametrize("V", [4, 500, 30000])
def test_nothing_takes_part(V):
    N = 70
    z = torch.full((N, V), math.nan, device="cuda", dtype=torch.bfloat16)
    f = torch.full((N,), math.nan, device="cuda")
    t = torch.full((N,), -1, device="cuda")
    r = tokens.logprobs(z, t, entropy=True)
    assert not r.logp.any() and not r.lse.any() and not r.entropy.any()
    p = tokens.policy_loss(z, t, f, f, weight=None, entropy_coef=0.1, kl_coef=0.1, logp_ref=f)
    assert not p.stats.any() and not p.logp.any() and not p.dlogits.any()
    p = tokens.policy_loss(z, torch.zeros_like(t), f, f, weight=torch.zeros(N, device="cuda"))
    assert not p.stats.any() and not p.logp.any() and not p.dlogits.any()
    q = tokens.preference_loss(z, t, tokens.batch_major(2, N // 2), logp_ref=f)
    assert abs(float(q.loss) - math.log(2)) < 2 * U and not q.dlogits.any() and float(q.stats[7]) == 0
    for n, seq in ((0, tokens.batch_major(0, 0)), (0, tokens.batch_major(2, 0)), (0, tokens.packed(torch.zeros(3, dtype=torch.int64, device="cuda")))):
        z0, t0, f0 = z[:n], t[:n], f[:n]
        assert tokens.logprobs(z0, t0).logp.shape == (0,)
        assert not tokens.policy_loss(z0, t0, f0, f0).stats.any()
        q = tokens.preference_loss(z0, t0, seq)
        assert float(q.stats[6]) == seq.count // 2 and q.margins.shape == (seq.count // 2,)
        assert tokens.lambda_returns(f0, f0, seq)[0].shape == (0,)


def _sequences(layout, count, g, longest, spare=0):
    n = torch.randint(0, longest + 1, (count,), generator=g)
    n[torch.randint(0, count, (1,), generator=g)] = longest
    n = n.tolist()
    rows = rows_of(layout, count, longest, n)
    if layout == "packed":
        off = torch.tensor([0] + list(np.cumsum(n)), dtype=torch.int64)
        return rows, int(off[-1]) + spare, tokens.packed(off.cuda())
    make = tokens.batch_major if layout == "batch" else tokens.time_major
    return rows, count * longest, make(count, longest, lengths=torch.tensor(n, dtype=torch.int32, device="cuda"))


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["packed", "batch", "time"])
@pytest.mark.parametrize("pairs,longest,V", [(1, 1, 5), (3, 9, 33), (2, 300, 7), (5, 20, 1031), (2, 13, 40001), (40, 3, 300), (1, 1500, 5), (3000, 2, 4)])
def test_preference_loss(dtype, layout, pairs, longest, V):
    g = torch.Generator().manual_seed(pairs * 31 + V)
    rows, N, seq = _sequences(layout, 2 * pairs, g, longest, spare=3)
    z, room, g = make_logits(N, V, dtype, 1, seed=2)
    before = room.clone()
    t = make_target(N, V, g, torch.int64, skip=0.2)
    x = ref_rows(z, t, 0.9)
    ref = (x["lp"] + 0.2 * torch.randn(N, generator=g)).float()
    label = torch.rand(pairs, generator=g)
    weight = torch.rand(pairs, generator=g) * (torch.arange(pairs) % 3 != 1)
    up = 256.0 * pairs if dtype == "fp16" else 1.0
    cu = lambda v: None if v is None else v.cuda()
    for mean, rf, y, w, margin, norm in ((False, ref, None, None, 0.0, 0.0), (True, None, label, weight, 0.5, 0.0), (False, ref, label, weight, -0.3, 7.0)):
        r = tokens.preference_loss(z, t, seq, beta=0.3, margin=margin, mean=mean, logp_ref=cu(rf), label=cu(y), weight=cu(w), norm=norm, scale=0.9, grad_scale=up)
        stats, h, g1, n = ref_preference(x, rows, 0.3, margin, mean, rf, y, w, norm)
        close(r.logp, x["lp"], U * x["lp"].abs() + 2 * roundings(V), "logp")
        # a sum of n log-probabilities is off by n times one of them at most
        per = 2 * roundings(V) * (1 if mean else longest) * 0.6 + U
        close(r.margins, h, per + U * np.abs(h), "margins")
        st = torch.tensor(stats, dtype=torch.float64)
        scale = max(1.0, (float(w.sum()) / norm) if norm else 1.0)
        close(r.stats[[0, 2, 3, 4, 5, 6, 7]], st[[0, 2, 3, 4, 5, 6, 7]], 2 * (per * scale + U * st[[0, 2, 3, 4, 5, 6, 7]].abs()), "stats")
        near = float((np.abs(h) <= per).sum())                    # pairs whose h the roundings may carry across 0
        assert abs(float(r.stats[1]) - stats[1]) <= 2 * U * max(1.0, abs(stats[1])) + (near if near else 0.0)      # (rounded to fp32: u of its size)
        want, size = ref_gradient(x, g1 * up, torch.zeros(N).double(), 0.9)
        close_gradient(r.dlogits, want, (1 + longest) * size, V, DT[dtype])
    assert torch.equal(room, before)
    own = room.clone()
    again = tokens.preference_loss(own[:, :V], t, seq, beta=0.3, margin=-0.3, logp_ref=ref.cuda(), label=label.cuda(), weight=weight.cuda(), norm=7.0, scale=0.9, grad_scale=up,
                                   out=own[:, :V])
    assert torch.equal(again.dlogits, r.dlogits) and torch.equal(again.stats, r.stats) and torch.equal(own[:, V:], room[:, V:])
    alone = tokens.preference_loss(z, t, seq, beta=0.3, margin=-0.3, logp_ref=ref.cuda(), label=label.cuda(), weight=weight.cuda(), norm=7.0, scale=0.9, gradient=False)
    assert alone.dlogits is None and torch.equal(alone.stats, r.stats)


@gpu
@pytest.mark.parametrize("value", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["packed", "batch", "time"])
@pytest.mark.parametrize("count,longest", [(1, 1), (3, 5), (70, 3), (2, 700), (1, 5000), (300, 40), (5, 2049), (1, 70001), (64, 513), (1030, 17), (8300, 300), (20000, 5), (100, 2000), (5000, 2)])
def test_lambda_returns(value, layout, count, longest):
    g = torch.Generator().manual_seed(count + longest)
    rows, N, seq = _sequences(layout, count, g, longest, spare=5)
    reward, v = torch.randn(N, generator=g), torch.randn(N, generator=g).to(DT[value])
    done, boot = (torch.rand(N, generator=g) < 0.05).to(torch.uint8), torch.randn(count, generator=g)
    for gamma, lam, d, b in ((1.0, 1.0, None, None), (0.99, 0.95, done, boot), (0.9, 0.0, None, boot), (0.0, 0.5, done, None), (1.0, 1.0, None, boot)):
        adv, ret = tokens.lambda_returns(reward.cuda(), v.cuda(), seq, gamma=gamma, lam=lam, done=None if d is None else d.cuda(), bootstrap=None if b is None else b.cuda())
        a, r = ref_returns(reward, v, rows, gamma, lam, d, b)
        # 64-bit sums, rounded once; where advantage and value cancel, the sum's own roundings (2^-52 of at most `longest` terms of size 4) remain
        close(adv, a, U * np.abs(a) + 8.0 * longest * longest * 2.0 ** -52, "adv")
        close(ret, r, U * np.abs(r) + 8.0 * longest * longest * 2.0 ** -52, "ret")


@gpu
def test_broken_sequences_stay_inside_the_rows():
    N, V, spare = 50, 40, 64
    room = torch.full((N + 2 * spare,), -7.0, device="cuda")
    grad = torch.full((N + 2 * spare, V), -7.0, device="cuda")
    z, _, g = make_logits(N, V, "fp32")
    t = make_target(N, V, g)
    for off in ([0, 60, 10, 20, 50], [-5, 10, 20, 30, 40], [0, 10, 5, 1 << 40, 50], [50, 40, 30, 20, 10]):
        seq = tokens.packed(torch.tensor(off, dtype=torch.int64, device="cuda"))
        q = tokens.preference_loss(z, t, seq, out=grad[spare:spare + N])
        assert torch.isnan(q.loss), off
        assert (grad[:spare] == -7).all() and (grad[spare + N:] == -7).all()
        L = binding.load()
        adv, ret = room.clone(), room.clone()
        ws = torch.empty(L.anakin_returns_workspace_bytes(N, 4), dtype=torch.uint8, device="cuda")
        r, v = torch.randn(N, device="cuda"), torch.randn(N, device="cuda")
        a = binding.ReturnsArgs(N, r.data_ptr(), v.data_ptr(), None, None, 0, 1.0, 0.9, adv[spare:].data_ptr(), ret[spare:].data_ptr())
        s = binding.SequenceArgs(0, 4, 0, seq.offsets.data_ptr(), None)
        assert L.anakin_lambda_returns(s, a, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        for x in (adv, ret):
            assert (x[:spare] == -7).all() and (x[spare + N:] == -7).all()
    for make in (tokens.batch_major, tokens.time_major):
        seq = make(10, 5, lengths=torch.tensor([5, 9, -3, 1 << 30, 0, 5, 5, 5, 5, 5], dtype=torch.int32, device="cuda"))
        assert torch.isnan(tokens.preference_loss(z, t, seq).loss)
        adv, _ = tokens.lambda_returns(room[:N].contiguous(), room[:N].contiguous(), seq)
        assert torch.isfinite(adv).all()


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [3, 70, 700, 5001, 70000])
@pytest.mark.parametrize("begin,to", [(1, 1), (3, 0), (5, 2), (7, 7)])
def test_rows_that_begin_anywhere(dtype, V, begin, to):
    """Logits and gradients a few elements off their allocations' starts, alike and not: the formulas hold, and nothing around the
    rows is written."""
    N = 5
    z, _, g = make_logits(N, V, dtype, seed=6)
    buf, back = torch.full((N * V + 16,), 7.0, dtype=DT[dtype], device="cuda"), torch.full((N * V + 16,), 7.0, dtype=DT[dtype], device="cuda")
    zb, out = buf[begin:begin + N * V].view(N, V), back[to:to + N * V].view(N, V)
    zb.copy_(z)
    before = buf.clone()
    t = make_target(N, V, g)
    t[2] = -1
    x = ref_rows(zb, t, 1.0)
    old, adv = (x["lp"] - 0.05).float(), torch.randn(N, generator=g)
    p = tokens.policy_loss(zb, t, old.cuda(), adv.cuda(), entropy_coef=0.02, out=out)
    _, g1, g2, on, size = ref_policy(x, old, adv, 0.2, 0.2, 0.0, None, 0.02, None, 0.0)
    close_gradient(p.dlogits, ref_gradient(x, g1, g2, 1.0)[0], 3 * ref_gradient(x, size, g2, 1.0)[1], V, DT[dtype])
    r = tokens.logprobs(zb, t)
    close_logp(r, x, V)
    d = tokens.logprobs_backward(zb, t, r.lse, adv.cuda(), out=out)
    want, size = ref_gradient(x, adv.double(), torch.zeros(N).double(), 1.0)
    close_gradient(d, want, size * (1 + x["lse"].abs()[:, None]), V, DT[dtype])
    assert torch.equal(buf, before) and (back[:to] == 7).all() and (back[to + N * V:] == 7).all()


@gpu
@pytest.mark.parametrize("rows,dtype,V", [(257, "fp32", 32769), (300, "fp32", 50001), (300, "fp32", 59392), (300, "fp32", 59399), (257, "bf16", 65537), (300, "fp16", 100003), (300, "bf16", 118791),
                                          (20, "fp32", 50001), (20, "fp32", 65600), (20, "fp32", 102400), (20, "fp32", 102411), (20, "bf16", 131080), (20, "fp16", 204800), (20, "bf16", 220007)])
def test_long_rows_of_the_clipped_loss(rows, dtype, V):
    """Rows on both sides of what registers and LDS hold, targets in every part of them; in place and not are alike; two calls too."""
    z, t, g = make_logits(12, V, dtype, seed=8)
    z[:, ::97] = -math.inf
    t = torch.tensor([1, 5, V - 1, V - 2, V // 2, 16384, V * 3 // 4, V - 600, 60, V // 3, V - 5000, 20001], device="cuda")
    z[torch.arange(12, device="cuda"), t] = 1.0
    at = torch.arange(12, device="cuda") * (rows // 13) + 1
    stride = V + 3
    buf = torch.full((rows * stride,), math.nan, dtype=DT[dtype], device="cuda")
    zb = buf.as_strided((rows, V), (stride, 1))
    zb[at] = z.cuda()
    tg = torch.full((rows,), -1, device="cuda")
    tg[at] = t
    x = ref_rows(z.cuda(), t, 1.0)
    adv = torch.randn(12, generator=g)
    old, ref = (x["lp"] - 0.05 * torch.randn(12, generator=g)).float(), (x["lp"] + 0.3).float()
    spread = lambda v: torch.zeros(rows, device="cuda").index_copy(0, at, v.cuda())
    call = lambda out=None: tokens.policy_loss(zb, tg, spread(old), spread(adv), kl_coef=0.1, logp_ref=spread(ref), entropy_coef=0.02, out=out)
    p, again = call(), call()
    stats, g1, g2, on, size = ref_policy(x, old, adv, 0.2, 0.2, 0.1, ref, 0.02, None, 0.0)
    close_gradient(p.dlogits[at], ref_gradient(x, g1, g2, 1.0)[0], 3 * ref_gradient(x, size, g2, 1.0)[1], V, DT[dtype])
    close(p.logp[at], x["lp"], U * x["lp"].abs() + 2 * roundings(V), "logp")
    close(p.stats, torch.tensor(stats, dtype=torch.float64), 4 * (1 + torch.tensor(stats).double().abs() + 3) * roundings(V), "stats")
    off = torch.ones(rows, dtype=torch.bool, device="cuda")
    off[at] = False
    assert not p.dlogits[off].any() and not p.logp[off].any()
    assert torch.equal(p.dlogits, again.dlogits) and torch.equal(p.stats, again.stats)
    q = call(out=zb)
    assert torch.equal(q.dlogits, p.dlogits) and torch.equal(q.stats, p.stats)
    gaps = buf.as_strided((rows - 1, 3), (stride, 1), V)
    assert torch.isnan(gaps).all()


@gpu
@pytest.mark.parametrize("layout,count,length", [("packed", 1, 2100000), ("packed", 1, 2097153), ("packed", 3, 1500000), ("batch", 2, 1100001), ("batch", 1, 5000000), ("time", 1, 2200000),
                                                 ("time", 2, 2100000), ("time", 7, 600000), ("time", 33, 33000), ("time", 40, 50001), ("time", 300, 35000)])
def test_very_long_sequences(layout, count, length):
    """gamma = lambda = 1 and numbers of 1/1024: every sum is exact in 64 bits, so returns and advantages are the rounded exact ones."""
    g = torch.Generator().manual_seed(count)
    N = count * length
    r, v = (torch.randint(-2048, 2049, (N,), generator=g) / 1024 for _ in range(2))
    done = (torch.rand(N, generator=g) < 2.0 / length).to(torch.uint8)
    boot = torch.randint(-2048, 2049, (count,), generator=g) / 1024
    lengths = torch.full((count,), length, dtype=torch.int32)
    if count > 1:
        lengths[0], lengths[1] = length - 777, length // 2
    if layout == "packed":
        seq = tokens.packed(torch.tensor([0] + lengths.cumsum(0).tolist(), device="cuda"))
    else:
        seq = (tokens.batch_major if layout == "batch" else tokens.time_major)(count, length, lengths.cuda())
    adv, ret = tokens.lambda_returns(r.cuda(), v.cuda(), seq, gamma=1.0, lam=1.0, done=done.cuda(), bootstrap=boot.cuda())
    want, member = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.bool)
    for s, rows in enumerate(rows_of(layout, count, length, lengths.tolist())):
        x, d = r[rows].double(), done[rows].bool()
        member[rows] = True
        ends = (torch.nonzero(d)[:, 0] + 1).tolist()
        at = 0
        for e in ends + [len(rows)]:
            part = torch.flip(torch.cumsum(torch.flip(x[at:e], [0]), 0), [0])
            want[rows[at:e]] = part + (0.0 if e in ends else float(boot[s]))
            at = e
    assert torch.equal(ret.cpu(), want.float())
    assert torch.equal(adv.cpu(), torch.where(member, want - v.double(), 0.0).float())


@gpu
@pytest.mark.parametrize("V", [6, 300, 9000])
def test_a_pair_with_an_impossible_token(V):
    """A forbidden target, and a row that allows nothing: the log-probability of their sequence is minus infinity; the gradient stays
    finite, and is zero where nothing is allowed."""
    z, _, g = make_logits(8, V, "fp32")
    t = make_target(8, V, g)
    z[1, int(t[1])] = -math.inf
    z[6] = -math.inf
    r = tokens.preference_loss(z, t, tokens.batch_major(4, 2))
    assert r.logp[1] == -math.inf and r.logp[6] == -math.inf
    assert r.margins[0] == -math.inf and r.margins[1] == math.inf and r.loss == math.inf
    assert torch.isfinite(r.dlogits).all() and not r.dlogits[6].any() and r.dlogits[0].any()
    lost = tokens.policy_loss(z, t, torch.zeros(8, device="cuda"), torch.ones(8, device="cuda"), entropy_coef=0.1)
    assert torch.isfinite(lost.stats).all() and torch.isfinite(lost.dlogits).all() and not lost.dlogits[6].any()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_beyond_32_bits(dtype):
    V, stride = 70000, (1 << 31) + 24                             # elements from row to row
    z, _, g = make_logits(3, V, dtype)
    room = torch.empty(2 * stride + V, dtype=DT[dtype], device="cuda")
    far = torch.as_strided(room, (3, V), (stride, 1))
    far.copy_(z)
    t = make_target(3, V, g)
    f = torch.randn(3, generator=g).cuda()
    a, b = tokens.logprobs(z, t, entropy=True), tokens.logprobs(far, t, entropy=True)
    assert torch.equal(a.logp, b.logp) and torch.equal(a.entropy, b.entropy)
    want = tokens.policy_loss(z, t, a.logp, f, entropy_coef=0.1)
    got = tokens.policy_loss(far, t, a.logp, f, entropy_coef=0.1, out=far)
    assert torch.equal(want.dlogits, got.dlogits) and torch.equal(want.stats, got.stats)


def _train_like(z, t, seq, reward, value, label):
    """The operators as a training program uses them together: scores, advantages, the clipped loss, the loss over pairs."""
    s = tokens.logprobs(z, t, entropy=True)
    adv, ret = tokens.lambda_returns(reward, value, seq, gamma=1.0, lam=0.95)
    p = tokens.policy_loss(z, t, s.logp * 0.98, adv, kl_coef=0.05, logp_ref=s.logp * 1.02, entropy_coef=0.01)
    q = tokens.preference_loss(z, t, seq, logp_ref=s.logp * 1.01, label=label)
    d = tokens.logprobs_backward(z, t, s.lse, adv, entropy=s.entropy, grad_entropy=ret)
    return [s.logp, s.lse, s.entropy, adv, ret, p.stats, p.logp, p.dlogits, q.stats, q.margins, q.dlogits, d]


@gpu
@pytest.mark.parametrize("N,V,dtype", [(40, 33, "fp32"), (96, 5003, "bf16"), (10, 140001, "fp16")])
def test_captured_together_and_replayed(N, V, dtype):
    z, _, g = make_logits(N, V, dtype, seed=3)
    t = make_target(N, V, g, skip=0.1)
    off = torch.tensor([0, N // 4, N // 2, N // 2 + 1, N], dtype=torch.int64, device="cuda")
    seq = tokens.packed(off)
    reward, value, label = torch.randn(N, generator=g).cuda(), torch.randn(N, generator=g).cuda(), torch.rand(2, generator=g).cuda()
    eager = [v.clone() for v in _train_like(z, t, seq, reward, value, label)]
    again = _train_like(z, t, seq, reward, value, label)
    assert all(torch.equal(a, b) for a, b in zip(eager, again))            # no result hangs on scheduling
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = _train_like(z, t, seq, reward, value, label)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, on_side))
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(_train_like(z, t, seq, reward, value, label))
        graphs.append(gr)
    z2, _, _ = make_logits(N, V, dtype, seed=4)
    first = z.clone()
    for k in range(4):
        z.copy_(z2 if k % 2 else first)
        graphs[0].replay(); graphs[1].replay()
        want = _train_like(z, t, seq, reward, value, label)
        torch.cuda.synchronize()
        for o in outs:
            assert all(torch.equal(a, b) for a, b in zip(want, o)), k


@gpu
def test_two_calls_at_once():
    z, _, g = make_logits(64, 9001, "bf16")
    t = make_target(64, 9001, g)
    f = torch.randn(64, generator=g).cuda()
    want = tokens.policy_loss(z, t, f - 9, f, entropy_coef=0.1)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for k in range(6):
        with torch.cuda.stream(a if k % 2 else b):
            got.append(tokens.policy_loss(z, t, f - 9, f, entropy_coef=0.1))
    torch.cuda.synchronize()
    for r in got:
        assert torch.equal(r.dlogits, want.dlogits) and torch.equal(r.stats, want.stats)


@gpu
def test_python_refusals_on_the_gpu():
    z = torch.zeros(4, 6, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    f = torch.zeros(4, device="cuda")
    bad = [lambda: tokens.logprobs(z.t(), t), lambda: tokens.logprobs(z[None], t), lambda: tokens.logprobs(z.double(), t), lambda: tokens.logprobs(z, t.float()),
           lambda: tokens.logprobs(z, t[:3]), lambda: tokens.logprobs(z, t.cpu()), lambda: tokens.logprobs(z, t, scale=0.0), lambda: tokens.logprobs(z[:, ::2], t),
           lambda: tokens.policy_loss(z, t, f.double(), f), lambda: tokens.policy_loss(z, t, f, None), lambda: tokens.policy_loss(z, t, f, f[:2]),
           lambda: tokens.policy_loss(z, t, f, f, kl_coef=0.1), lambda: tokens.policy_loss(z, t, f, f, clip=(-0.1, 0.2)),
           lambda: tokens.policy_loss(z, t, f, f, out=z.half()), lambda: tokens.policy_loss(z, t, f, f, out=z[:3]), lambda: tokens.policy_loss(z, t, f, f, weight=torch.zeros(8, device="cuda")[::2]),
           lambda: tokens.logprobs_backward(z, t, f, f, grad_entropy=f), lambda: tokens.preference_loss(z, t, tokens.batch_major(2, 3)),
           lambda: tokens.preference_loss(z, t, tokens.batch_major(1, 4)), lambda: tokens.preference_loss(z, t, 5), lambda: tokens.preference_loss(z, t, tokens.batch_major(2, 2), label=f),
           lambda: tokens.lambda_returns(f, f, tokens.batch_major(3, 3)), lambda: tokens.lambda_returns(f, t, tokens.batch_major(2, 2)),
           lambda: tokens.lambda_returns(f, f, tokens.batch_major(2, 2), gamma=2.0), lambda: tokens.lambda_returns(f, f, tokens.batch_major(2, 2), done=t)]
    for k, call in enumerate(bad):
        with pytest.raises(binding.AnakinError):
            call()
            assert False, k
    room = torch.zeros(4, 8, device="cuda")
    with pytest.raises(binding.AnakinError):                        # overlaps without being the same rows
        tokens.policy_loss(room[:, :6], t, f, f, out=room[:, 1:7])
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["packed", "batch", "time"])
@pytest.mark.parametrize("V", [5, 70, 300, 1031, 5001, 70001])
def test_rows_outside_the_pairs_may_hold_anything(dtype, layout, V):
    """Rows in no sequence and rows of pairs of weight 0 get zeros, whatever their logits and references hold; the other rows' gradient
    and the loss are those of ordinary numbers in their place, in place too."""
    n, length = [3, 1, 4, 0, 2, 3], 4
    rows = rows_of(layout, 6, length, n)
    N = 24 if layout != "packed" else sum(n) + 5
    if layout == "packed":
        seq = tokens.packed(torch.tensor([0] + list(np.cumsum(n)), device="cuda"))
    else:
        seq = (tokens.batch_major if layout == "batch" else tokens.time_major)(6, length, torch.tensor(n, dtype=torch.int32, device="cuda"))
    z, room, g = make_logits(N, V, dtype, 1, seed=9)
    t = make_target(N, V, g)
    ref, label, weight = torch.randn(N, generator=g).cuda(), torch.rand(3, generator=g).cuda(), torch.tensor([1.0, 0.0, 0.5], device="cuda")
    on = np.zeros(N, bool)
    for s in (0, 2, 3, 5):
        on[rows[s]] = True
    off = torch.tensor(~on, device="cuda")
    call = lambda x, r, **kw: tokens.preference_loss(x, t, seq, beta=0.7, logp_ref=r, label=label, weight=weight, **kw)
    want = call(z, ref)
    assert not want.dlogits[off].any() and want.dlogits[~off].any()
    x, bad = room.clone(), ref.clone()
    bad[off] = math.nan
    for k, i in enumerate(torch.nonzero(off)[:, 0].tolist()):
        x[i, :V] = [math.nan, math.inf, -math.inf][k % 3]
        x[i, k % V] = [math.nan, -math.inf, math.inf, 1.0][k % 4]
    got = call(x[:, :V], bad)
    assert torch.equal(got.stats, want.stats) and torch.equal(got.dlogits, want.dlogits)
    own = x.clone()
    again = call(own[:, :V], bad, out=own[:, :V])
    assert torch.equal(again.dlogits, want.dlogits) and torch.equal(again.stats, want.stats) and torch.equal(own[:, V:], x[:, V:])


@gpu
@pytest.mark.parametrize("V", [5, 70, 300, 1031, 5001, 70001])
def test_no_weight_means_no_gradient(V):
    """Weights that cancel: W = 0 gives loss and gradient 0, also where a ratio overflows, a logit is a NaN or a sequence impossible."""
    N = 8
    z, _, g = make_logits(N, V, "fp32")
    t = make_target(N, V, g)
    w = torch.tensor([1.0, -1.0] * (N // 2), device="cuda")
    adv = torch.randn(N, generator=g).cuda()
    old = torch.zeros(N, device="cuda")
    old[1] = -2e3
    for poison in (False, True):
        if poison:
            z[3, V - 1] = math.nan
        r = tokens.policy_loss(z, t, old, adv, entropy_coef=0.1, weight=w)
        assert not r.stats[:7].any() and float(r.stats[7]) == N and not r.dlogits.any()
        q = tokens.preference_loss(z, t, tokens.batch_major(4, 2), weight=w[:2])
        assert not q.stats[:6].any() and not q.dlogits.any()


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [2, 9, 64, 300, 1030, 5000, 33000, 132000])
@pytest.mark.parametrize("scale", [1.0, 1.25, 0.7, 0.37])
def test_backward_pass_of_masks_and_extremes(dtype, V, scale):
    """Every row of the kinds above, whose log-sum-exp may be past what binary32 tells probabilities from, or past its range."""
    z, t = _special(dtype, V)
    g = torch.Generator().manual_seed(2)
    base = torch.randn(V, generator=g)
    more = torch.stack([base + o for o in (900.0, -1500.0, 2e4, -6e4 if dtype == "fp16" else -3e7)]).to(DT[dtype])
    z, t = torch.cat([z, more, more]), torch.cat([t, torch.tensor([0, V - 1, V // 2, 0, V - 1, 0, V // 3, -1])])
    x = ref_rows(z, t, scale)
    N = len(t)
    zc, tc = z.cuda(), t.cuda()
    r = tokens.logprobs(zc, tc, scale=scale, entropy=True)
    g1, g2 = 64 * torch.randn(N, generator=g), 64 * torch.rand(N, generator=g)
    for e in (None, g2):
        d = tokens.logprobs_backward(zc, tc, r.lse, g1.cuda(), entropy=r.entropy, grad_entropy=None if e is None else e.cuda(), scale=scale)
        want, size = ref_gradient(x, g1.double(), torch.zeros(N).double() if e is None else e.double(), scale)
        # from the handed-over lse, rounded to fp32, as long as it is below 2^10; beyond from the row's own sums
        lse = x["lse"].abs().nan_to_num(0, 0, 0)
        close_gradient(d, want, size * (1 + torch.where(lse < 1024, lse, 0.0))[:, None], V, DT[dtype])
        assert torch.isfinite(d).all()
        own = torch.full((N, V + 1), 7.0, dtype=DT[dtype], device="cuda")
        own[:, :V] = zc
        again = tokens.logprobs_backward(own[:, :V], tc, r.lse, g1.cuda(), entropy=r.entropy, grad_entropy=None if e is None else e.cuda(), scale=scale, out=own[:, :V])
        close_gradient(again, want, size * (1 + torch.where(lse < 1024, lse, 0.0))[:, None], V, DT[dtype])
        assert (own[:, V] == 7).all()


@gpu
def test_a_broken_pair_without_weight_is_reported():
    z, _, g = make_logits(50, 40, "fp32")
    t = make_target(50, 40, g)
    for seq in (tokens.packed(torch.tensor([0, 5, 3, 8, 50], device="cuda")), tokens.batch_major(4, 12, torch.tensor([12, 13, 3, 4], dtype=torch.int32, device="cuda")),
                tokens.time_major(4, 12, torch.tensor([12, 12, 3, -1], dtype=torch.int32, device="cuda"))):
        n = 50 if seq.offsets is not None else 48
        for w in ([1.0, 0.0], [0.0, 0.0]):
            q = tokens.preference_loss(z[:n], t[:n], seq, weight=torch.tensor(w, device="cuda"))
            assert torch.isnan(q.loss), (seq.layout, w)


def test_logits_that_record_gradients_are_refused():
    z = torch.zeros(3, 5, requires_grad=True)
    t, f = torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    for call in (lambda x: tokens.logprobs(x, t), lambda x: tokens.policy_loss(x, t, f, f), lambda x: tokens.preference_loss(x, t, tokens.batch_major(1, 3))):
        for x in (z, z * 2):
            with pytest.raises(binding.AnakinError, match="detach"):
                call(x)
        for x in (z.detach(), z):                                  # (these get as far as the device)
            with torch.no_grad(), pytest.raises(RuntimeError, match="GPU"):
                call(x)


@gpu
def test_gradients_in_place_are_seen_by_autograd():
    leaf = torch.randn(4, 7, device="cuda", requires_grad=True)
    t, f = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, device="cuda")
    lse = tokens.logprobs(leaf.detach(), t).lse
    for call in (lambda z: tokens.policy_loss(z, t, f, f, out=z), lambda z: tokens.preference_loss(z, t, tokens.batch_major(2, 2), out=z), lambda z: tokens.logprobs_backward(z, t, lse, f, out=z)):
        logits = leaf * 1.0
        other = logits.square().sum()                              # keeps the logits for its backward pass
        call(logits.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            other.backward()
        with pytest.raises(binding.AnakinError):                   # an `out` whose history would be lost
            tokens.policy_loss(logits.detach(), t, f, f, out=torch.zeros(4, 7, device="cuda", requires_grad=True))
    # the pattern that the documentation names
    logits = leaf * 1.0
    r = tokens.policy_loss(logits.detach(), t, f, f + 1.0)
    logits.backward(r.dlogits)
    assert torch.equal(leaf.grad, r.dlogits)
    with torch.inference_mode():
        z = torch.randn(4, 7, device="cuda")
        tokens.policy_loss(z, t, f, f, out=z)


# ---- accuracy: bounds that the arithmetic kept for it can hold, and no other ----------------------------------------------
# The exponential instruction is good to one step, 2^-23 of its value; a quarter of that is allowed it as a mean over many rows.
EXP_MEAN = 2.0 ** -25


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [4, 32, 64, 512, 1024, 4096, 32768])
@pytest.mark.parametrize("scale", [1.0, 0.7, 1.25])
def test_pairs_do_not_see_a_number_added_to_a_row(dtype, V, scale):
    """Logits on a grid, and the same with 4 more in every column: their distances to the maximum are the same numbers, so are the
    log-probabilities, to the last bit (with the exponents' own roundings lost they would differ by some 1e-8 a row), and h is 0."""
    n = 24
    g = torch.Generator().manual_seed(V)
    z = torch.randint(-12, 13, (n, V), generator=g) / 8.0         # up to 5.5 on steps of 1/8: 6 bits, which every type has
    t = torch.randint(0, V, (n,), generator=g)
    both = torch.cat([z, z + 4.0]).to(DT[dtype]).cuda()
    assert torch.equal(both[:n].cpu().double() + 4.0, both[n:].cpu().double())
    q = tokens.preference_loss(both, torch.cat([t, t]).cuda(), tokens.batch_major(2, n), beta=1.0, scale=scale)
    assert float(q.margins[0]) == 0.0 and torch.equal(q.logp[:n], q.logp[n:])
    assert torch.equal(q.dlogits[:n] == 0, q.dlogits[n:] == 0) and q.dlogits.any()


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V,n", [(3, 40000), (64, 20000), (1000, 8000), (8000, 1500), (40000, 400)])
@pytest.mark.parametrize("scale", [0.7, 1.25, 0.79])
def test_log_probabilities_have_no_drift(dtype, V, n, scale):
    """Means over many rows, where roundings average out.  What is left is the exponential's own, n EXP_MEAN, and 6 times the root of
    n roundings: for a sum of a pair's rows one of 2^-24 each, for outputs in fp32 one of U |logp|.  (scale log2 e rounded to fp32 is
    off by up to 2^-24 of itself, at 0.79 by 5e-8: a mean logit of 25 turns that into 30 times EXP_MEAN if it is not put back.)"""
    g = torch.Generator(device="cuda").manual_seed(V)
    z = (torch.randn(n, V, generator=g, device="cuda") * 2.5 + 24.0).to(DT[dtype])
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    lp = torch.empty(n, dtype=torch.float64)
    for i in range(0, n, 2000):
        x = z[i:i + 2000].cpu().double() * scale
        m = x.max(1, keepdim=True).values
        lp[i:i + 2000] = (x.gather(1, t[i:i + 2000].cpu()[:, None]) - m - torch.log(torch.exp(x - m).sum(1, keepdim=True)))[:, 0]
    r = tokens.logprobs(z, t, scale=scale)
    off = float((r.logp.cpu().double() - lp).mean())
    assert abs(off) <= EXP_MEAN + 6 * U * float(lp.abs().max()) / math.sqrt(n), off
    # (the margin takes h to 0, so that fp32 holds what is off)
    q = tokens.preference_loss(z, t, tokens.packed(torch.tensor([0, n, n], device="cuda")), beta=1.0, margin=float(lp.sum()), scale=scale, gradient=False)
    assert abs(float(q.margins[0])) <= n * EXP_MEAN + 6 * math.sqrt(n) * U, float(q.margins[0])


@gpu
@pytest.mark.parametrize("V,n", [(32768, 96), (131072, 64), (200003, 32)])
def test_long_rows_add_up(V, n):
    """Rows shifted to a log-sum-exp near 0, where fp32 holds it to 2^-30: root of the mean square of what it is off.  EXP_MEAN, and as
    much for sums: a thread's chain of up to 64 additions, 2^-24 sqrt(64) / 2, over 256 threads at least, and their joins."""
    g = torch.Generator().manual_seed(V)
    z = torch.randn(n, V, generator=g) * 2.5
    z = z - torch.logsumexp(z.double(), 1).float()[:, None] + torch.rand(n, 1, generator=g) * 0.02 - 0.01
    t = torch.zeros(n, dtype=torch.int64)
    off = tokens.logprobs(z.cuda(), t.cuda()).lse.cpu().double() - torch.logsumexp(z.double(), 1)
    assert float((off ** 2).mean().sqrt()) <= 2 * EXP_MEAN


@gpu
def test_ratios_are_rounded_once():
    """One column: the log-probability is 0, and the ratio e^-old rounded to fp32."""
    z, t, one = torch.zeros(1, 1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, device="cuda")
    for i in range(60):
        old = torch.tensor([1.0 - 0.21 * i])
        r = tokens.policy_loss(z, t, old.cuda(), one, clip=(1.0, 1e6), gradient=False)
        want = math.exp(-float(old[0]))
        assert abs(float(r.stats[5]) - want) <= (U + 2.0 ** -36) * want and abs(float(r.loss) + want) <= (U + 2.0 ** -36) * want


@gpu
@pytest.mark.parametrize("layout", ["packed", "batch", "time"])
def test_share_of_pairs_the_first_wins(layout):
    """The weighted share of pairs with h > 0, where no h is near 0 nor a sequence empty."""
    pairs, n, V = 500, 3, 40
    z, _, g = make_logits(2 * pairs * n, V, "fp32", seed=11)
    t = make_target(2 * pairs * n, V, g)
    seq = tokens.packed(torch.arange(0, 2 * pairs * n + 1, n, device="cuda")) if layout == "packed" else (tokens.batch_major if layout == "batch" else tokens.time_major)(2 * pairs, n)
    rows = rows_of(layout, 2 * pairs, n, [n] * (2 * pairs))
    weight = torch.rand(pairs, generator=g)
    stats, h, _, _ = ref_preference(ref_rows(z, t, 1.0), rows, 0.5, 0.3, False, None, None, weight, 0.0)
    near = np.abs(h) < 1e-4
    weight[torch.tensor(near)] = 0.0
    assert near.sum() < 5
    want = float((weight.double().numpy() * (h > 0)).sum() / weight.double().sum())
    q = tokens.preference_loss(z, t, seq, beta=0.5, margin=0.3, weight=weight.cuda())
    assert abs(float(q.stats[1]) - want) <= 1.01 * U * want and 0.2 < want < 0.8
