"""Operators of token policies on torch tensors: log-probabilities of chosen columns of a matrix of logits, the clipped
policy loss, a loss over pairs of sequences, and lambda-returns over sequences of unequal length.

Argument marshalling only, like `binding`: PyTorch allocates outputs and workspace and provides the stream, all
arithmetic runs in libanakin's kernels, there is no fallback.  Everything runs on the current stream of the tensors'
device; nothing synchronises.  No gradients are recorded: a loss and its gradient towards the logits come from one call, and
all inputs but the logits are constants to it.  Logits that autograd follows would lose that history without a word, so they are
refused unless it is switched off (torch.no_grad): call with logits.detach() and hand the result to logits.backward(r.dlogits).

    logits      [rows][vocab], fp32, bf16 or fp16, columns adjacent, any distance from row to row
    target      [rows], uint8, int32 or int64: the chosen column; a row with a target outside [0, vocab) takes no part
    scale       softmax(scale * logits) is the policy (one over the sampling temperature)

Next-token targets of whole sequences are the tokens shifted by one, with -1 behind the last one of each sequence (and
where a prompt stands): logits are used where they lie, without a copy.
"""
import ctypes as C
from collections import namedtuple

import torch

from . import binding
from .binding import AnakinError, E_INVALID_ARG

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_INDEX = {torch.uint8: 0, torch.int32: 1, torch.int64: 2}
PACKED, BATCH, TIME = 0, 1, 2

LogProbs = namedtuple("LogProbs", "logp lse entropy")


class PolicyLoss(namedtuple("PolicyLoss", "stats logp dlogits")):
    """stats: loss, and weighted means of policy term, KL term, entropy, share of clipped rows, ratio; the weight they were
    divided by; rows that took part."""
    __slots__ = ()

    @property
    def loss(self):
        return self.stats[0]


class PreferenceLoss(namedtuple("PreferenceLoss", "stats margins logp dlogits")):
    """stats: loss, and weighted means of [h > 0], beta D_first, beta D_second, h; the weight they were divided by; pairs
    and tokens that took part."""
    __slots__ = ()

    @property
    def loss(self):
        return self.stats[0]


class Sequences:
    """Which rows the tokens of each sequence are; see packed, batch_major, time_major."""
    __slots__ = ("layout", "count", "length", "offsets", "lengths")

    def __init__(self, layout, count, length, offsets, lengths):
        self.layout, self.count, self.length, self.offsets, self.lengths = layout, int(count), int(length), offsets, lengths


def packed(offsets):
    """Sequence s is rows offsets[s] .. offsets[s + 1] - 1; offsets: int64 [count + 1], ascending, on the device."""
    if offsets.dtype != torch.int64 or offsets.dim() != 1 or offsets.numel() < 1:
        _refuse("offsets have to be int64 [count + 1]")
    return Sequences(PACKED, offsets.numel() - 1, 0, offsets, None)


def batch_major(count, length, lengths=None):
    """Token j of sequence s is row s * length + j, for j < lengths[s] (int32 [count] on the device; None: length)."""
    return Sequences(BATCH, count, length, None, _lengths(lengths, count))


def time_major(count, length, lengths=None):
    """Token j of sequence s is row j * count + s, for j < lengths[s] (int32 [count] on the device; None: length)."""
    return Sequences(TIME, count, length, None, _lengths(lengths, count))


def _lengths(lengths, count):
    if lengths is not None and (lengths.dtype != torch.int32 or tuple(lengths.shape) != (count,)):
        _refuse("lengths have to be int32 [count]")
    return lengths


def _refuse(why):
    raise AnakinError(E_INVALID_ARG, why)


class _Call:
    """The device and stream of one call, checks of its tensors, and the library's answer."""

    def __init__(self, first, recorded=False):
        if not isinstance(first, torch.Tensor):
            _refuse("a tensor is wanted")
        if recorded and first.requires_grad and torch.is_grad_enabled():
            _refuse("no history is recorded: pass logits.detach() and hand dlogits to logits.backward")
        if not first.is_cuda:
            raise RuntimeError("the operators of token policies run on the GPU alone")
        self.L = binding.load()
        self.device = first.device

    def vector(self, t, n, name, dtype=torch.float32, optional=True):
        """The address of a contiguous [n] tensor of the call's device."""
        if t is None:
            if not optional:
                _refuse(f"{name} is missing")
            return None
        if t.device != self.device:
            _refuse(f"{name} is on another device")
        if t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
            _refuse(f"{name} has to be contiguous {dtype} [{n}]")
        return t.data_ptr()

    def rows(self, logits, target, scale):
        if logits.dim() != 2 or logits.dtype not in _TYPES:
            _refuse("logits have to be [rows][vocab] of fp32, bf16 or fp16")
        n, v = logits.shape
        if v < 1 or (v > 1 and logits.stride(1) != 1):
            _refuse("the columns of the logits have to be adjacent")
        if target.dtype not in _INDEX:
            _refuse("targets have to be uint8, int32 or int64")
        stride = logits.stride(0) if n > 1 else v
        return binding.Rows(logits.data_ptr(), n, v, stride, self.vector(target, n, "target", target.dtype), _TYPES[logits.dtype], _INDEX[target.dtype], scale)

    def gradient(self, logits, out):
        """Where the gradient goes: `out` (it may be the logits), or a new tensor."""
        if out is None:
            out = torch.empty(logits.shape, dtype=logits.dtype, device=self.device)
        elif out.device != self.device or out.dtype != logits.dtype or out.shape != logits.shape or (out.shape[1] > 1 and out.stride(1) != 1):
            _refuse("out has to be like the logits: shape, type, device, adjacent columns")
        elif out.requires_grad and torch.is_grad_enabled():
            _refuse("out is written without history: pass out.detach()")
        elif not out.is_inference():
            torch.autograd.graph.increment_version(out)               # autograd's own copies of it are stale from here on
        return out, (out.stride(0) if out.shape[0] > 1 else out.shape[1])

    def sequences(self, q):
        if not isinstance(q, Sequences):
            _refuse("sequences come from packed, batch_major or time_major")
        return binding.SequenceArgs(q.layout, q.count, q.length, self.vector(q.offsets, q.count + 1, "offsets", torch.int64),
                                    self.vector(q.lengths, q.count, "lengths", torch.int32))

    def empty(self, n, dtype=torch.float32):
        return torch.empty(n, dtype=dtype, device=self.device)

    def run(self, function, *args):
        index = self.device.index
        stream = torch._C._cuda_getCurrentRawStream(index)             # the current stream's handle, without an object around it
        if torch.cuda.current_device() == index:
            rc = function(*args, stream)
        else:
            with torch.cuda.device(index):
                rc = function(*args, stream)
        if rc != binding.OK:
            raise AnakinError(rc, self.L.anakin_last_error(None).decode())


def logprobs(logits, target, scale=1.0, entropy=False):
    """(logp, lse, entropy or None), fp32 [rows]: log-probability of the target under softmax(scale * logits), log-sum-exp,
    entropy.  Rows that take no part get zeros."""
    c = _Call(logits, recorded=True)
    x = c.rows(logits, target, scale)
    logp, lse = c.empty(x.rows), c.empty(x.rows)
    h = c.empty(x.rows) if entropy else None
    c.run(c.L.anakin_token_logprobs, x, logp.data_ptr(), lse.data_ptr(), h.data_ptr() if entropy else None)
    return LogProbs(logp, lse, h)


def logprobs_backward(logits, target, lse, grad_logp, *, entropy=None, grad_entropy=None, scale=1.0, out=None):
    """d / d logits of sum grad_logp logp + sum grad_entropy entropy, in the logits' type; lse and entropy: of `logprobs`.
    out: where it goes (may be the logits themselves); None: a new tensor."""
    c = _Call(logits)
    x = c.rows(logits, target, scale)
    out, stride = c.gradient(logits, out)
    n = x.rows
    c.run(c.L.anakin_token_logprobs_backward, x, c.vector(lse, n, "lse", optional=False), c.vector(entropy, n, "entropy"),
          c.vector(grad_logp, n, "grad_logp", optional=False), c.vector(grad_entropy, n, "grad_entropy"), out.data_ptr(), stride)
    return out


def policy_loss(logits, target, logp_old, adv, *, clip=0.2, kl_coef=0.0, logp_ref=None, entropy_coef=0.0, weight=None, norm=0.0, scale=1.0,
                grad_scale=1.0, gradient=True, out=None):
    """Clipped policy loss, l = -min(r A, clip(r, 1 - low, 1 + high) A) + kl_coef (e^d - d - 1) - entropy_coef H with
    r = exp(logp - logp_old), d = logp_ref - logp; the weighted mean over the rows that take part, and grad_scale times its
    gradient towards the logits.  clip: one width or (low, high).  norm: divide by this in place of the sum of the weights.
    gradient=False: the loss alone.  out: where the gradient goes (may be the logits themselves)."""
    c = _Call(logits, recorded=True)
    x = c.rows(logits, target, scale)
    n = x.rows
    low, high = clip if isinstance(clip, (tuple, list)) else (clip, clip)
    stats, logp = c.empty(8), c.empty(n)
    out, stride = c.gradient(logits, out) if gradient else (None, 0)
    a = binding.PolicyArgs(c.vector(logp_old, n, "logp_old", optional=False), c.vector(adv, n, "adv", optional=False), c.vector(logp_ref, n, "logp_ref"),
                           c.vector(weight, n, "weight"), low, high, kl_coef, entropy_coef, norm, grad_scale, stats.data_ptr(), logp.data_ptr(),
                           out.data_ptr() if gradient else None, stride)
    ws = c.empty(c.L.anakin_rows_workspace_bytes(n, x.vocab, 0), torch.uint8)
    c.run(c.L.anakin_policy_loss, x, a, ws.data_ptr(), ws.numel())
    return PolicyLoss(stats, logp, out)


def preference_loss(logits, target, sequences, *, beta=0.1, margin=0.0, mean=False, logp_ref=None, label=None, weight=None, norm=0.0, scale=1.0,
                    grad_scale=1.0, gradient=True, out=None):
    """Loss over pairs of sequences (the first half of them with the second half, in order): -y log sigmoid(h) - (1 - y)
    log sigmoid(-h), h = beta (D_first - D_second) - margin, D the sum (mean: the mean) over a sequence's tokens of
    logp - logp_ref, y = label (None: 1, the first is the preferred one); the weighted mean over the pairs, and grad_scale
    times its gradient towards the logits.  margins: h of every pair."""
    c = _Call(logits, recorded=True)
    x = c.rows(logits, target, scale)
    q = c.sequences(sequences)
    n, pairs = x.rows, q.count // 2
    stats, margins, logp = c.empty(8), c.empty(pairs), c.empty(n)
    out, stride = c.gradient(logits, out) if gradient else (None, 0)
    a = binding.PreferenceArgs(c.vector(logp_ref, n, "logp_ref"), c.vector(label, pairs, "label"), c.vector(weight, pairs, "weight"), beta, margin, norm,
                               grad_scale, 1 if mean else 0, stats.data_ptr(), margins.data_ptr(), logp.data_ptr(), out.data_ptr() if gradient else None, stride)
    ws = c.empty(c.L.anakin_rows_workspace_bytes(n, x.vocab, max(1, pairs)), torch.uint8)
    c.run(c.L.anakin_preference_loss, x, q, a, ws.data_ptr(), ws.numel())
    return PreferenceLoss(stats, margins, logp, out)


def lambda_returns(reward, value, sequences, *, gamma=1.0, lam=1.0, done=None, bootstrap=None):
    """(adv, ret), fp32 [rows]: ret_t = r_t + disc_t ((1 - lam) V_{t+1} + lam ret_{t+1}), adv = ret - value; disc = gamma, 0
    where done is set; behind a sequence's last token both V and ret are bootstrap[s] (None: 0).  reward: fp32 [rows];
    value: fp32, bf16 or fp16 [rows]; done: uint8 [rows].  Rows in no sequence get zeros."""
    c = _Call(reward)
    n = reward.shape[0] if reward.dim() == 1 else _refuse("rewards have to be [rows]")
    if value.dtype not in _TYPES:
        _refuse("values have to be fp32, bf16 or fp16")
    q = c.sequences(sequences)
    adv, ret = c.empty(n), c.empty(n)
    a = binding.ReturnsArgs(n, c.vector(reward, n, "reward"), c.vector(value, n, "value", value.dtype, optional=False), c.vector(done, n, "done", torch.uint8),
                            c.vector(bootstrap, q.count, "bootstrap"), _TYPES[value.dtype], gamma, lam, adv.data_ptr(), ret.data_ptr())
    ws = c.empty(c.L.anakin_returns_workspace_bytes(n, q.count), torch.uint8)
    c.run(c.L.anakin_lambda_returns, q, a, ws.data_ptr(), ws.numel())
    return adv, ret
