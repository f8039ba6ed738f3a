"""A client's sensitivity map: ``Sensitivity(W, D_i)`` of Algorithm 1, Step 1 of Selective Parameter Encryption.

The map has a score for every parameter w of the model, the mean over the client's samples k of |d/dy_k (d loss / dw)|.  Under
cross entropy, loss_k = -sum_c y_{k,c} log p_c, the derivative by the coordinate of the sample's label is, up to its sign, the
gradient of the label's log probability; a sequence's is that of the sum over its tokens.  So a pass over a batch computes the tokens'
log probabilities, sends their gradient back through the model and, in every layer, takes the magnitudes of the samples' gradients,
which are never in memory one by one.

The map is laid out as the flattened model (``torch.nn.utils.parameters_to_vector(model.parameters())``), which is what he_pack and
he_encrypt take; the server's weighted sum of the clients' encrypted maps, decrypted, goes to he_select_mask.
"""
from __future__ import annotations

import contextlib
import threading
from typing import Dict, Iterable, List, NamedTuple, Optional, Tuple

import torch
from torch import nn

from . import (HE_ERR_INVALID_ARG, HE_OK, Ctx, HeError, _stream, he_ctx_status, he_layer_norm, he_layer_norm_backward, he_linear_sensitivity,
               he_token_log_probs, he_token_log_probs_backward)


class Sensitivity(NamedTuple):
    map: torch.Tensor        # float32 [P], 0 for parameters that are not trained
    samples: int
    tokens: int              # with a target
    log_prob: float          # mean over them
    entropy: float           # mean over all tokens


def _refuse(why: str) -> None:
    raise HeError(HE_ERR_INVALID_ARG, "sensitivity_map: " + why)


class _Part(NamedTuple):
    """A module's places in the map."""
    name: str
    weight: Optional[torch.Tensor]
    bias: Optional[torch.Tensor]


class _Pass:
    """What the layers of one batch's backward pass need."""

    def __init__(self, ctx: Ctx, count: int, device: torch.device):
        self.ctx, self.count, self.device = ctx, count, device
        self.offsets: Dict[int, Optional[torch.Tensor]] = {}
        self.seen: set = set()
        self.home = torch.cuda.current_stream(device) if device.type == "cuda" else None
        self.handle = self.home.cuda_stream if self.home else 0

    def samples(self, rows: int) -> Optional[torch.Tensor]:
        """Offsets of the batch's samples in a layer's rows (None: a row each)."""
        if rows not in self.offsets:
            self.offsets[rows] = None if rows == self.count else \
                torch.arange(0, rows + 1, rows // self.count, dtype=torch.int32, device=self.device) if rows else \
                torch.zeros(self.count + 1, dtype=torch.int32, device=self.device)
            if self.home and self.offsets[rows] is not None:
                self.offsets[rows].record_stream(self.home)      # other streams' uses are behind one another, and ahead of that one's
        return self.offsets[rows]

    # The pass backward goes by the streams that the layers ran on.  Work on the map, and on the samples' offsets, comes there behind what the pass's own
    # stream has to do, which goes on behind it.
    def begin(self) -> Optional[torch.cuda.Stream]:
        if _stream() == self.handle:
            return None
        stream = torch.cuda.current_stream()
        stream.wait_stream(self.home)
        return stream

    def end(self, stream: Optional[torch.cuda.Stream]) -> None:
        if stream is not None:
            self.home.wait_stream(stream)

    def enter(self, part: _Part, shape: torch.Size) -> None:
        if len(shape) < 2 or shape[0] != self.count:
            _refuse("layer %s is given the shape %s: its first dimension has to be that of the %d samples" % (part.name, tuple(shape), self.count))
        if not torch.is_grad_enabled():
            _refuse("layer %s is run under no_grad, where it gets no score; give its parameters requires_grad=False if that is meant" % part.name)
        if part.name in self.seen:
            _refuse("layer %s is used twice in a pass: its two gradients would have to be added before their magnitudes are" % part.name)
        self.seen.add(part.name)


def _rows(t: torch.Tensor) -> torch.Tensor:
    t = t.reshape(-1, t.shape[-1])
    return t if t.stride(1) == 1 or t.shape[1] == 1 else t.contiguous()


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, part, state):
        y = nn.functional.linear(x, weight, bias)
        ctx.save_for_backward(x.to(y.dtype), weight)         # under autocast the layer's type, not the input's
        ctx.part, ctx.state = part, state
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        part, state = ctx.part, ctx.state
        rows = _rows(x)
        stream = state.begin()
        he_linear_sensitivity(state.ctx, rows, _rows(dy), samples=state.samples(rows.shape[0]), out=part.weight, out_bias=part.bias, accumulate=True,
                              bias=part.bias is not None)
        state.end(stream)
        return dy @ weight.to(dy.dtype) if ctx.needs_input_grad[0] else None, None, None, None, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, part, state):
        rows, ctx.dtype = _rows(x), x.dtype
        # autocast computes and returns layer norms in fp32, those of 64 bits excepted
        if torch.is_autocast_enabled(x.device.type) and x.dtype != torch.float64:
            rows, weight, bias = (None if t is None else t.float() for t in (rows, weight, bias))
        y, mean, rstd = he_layer_norm(state.ctx, rows, weight, bias, eps)
        ctx.save_for_backward(rows, weight, mean, rstd)
        ctx.part, ctx.state, ctx.shape = part, state, x.shape
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        rows, weight, mean, rstd = ctx.saved_tensors
        part, state = ctx.part, ctx.state
        stream = state.begin()
        every = state.samples(rows.shape[0])
        if every is None:                                    # a row for each sample
            every = torch.arange(rows.shape[0] + 1, dtype=torch.int32, device=rows.device)
        dx, dweight, dbias = he_layer_norm_backward(state.ctx, _rows(dy), rows, mean, rstd, weight, samples=every)
        if part.weight is not None:
            part.weight.add_(dweight)
        if part.bias is not None:
            part.bias.add_(dbias)
        state.end(stream)
        return dx.view(ctx.shape).to(ctx.dtype), None, None, None, None, None


def _parts(model: nn.Module, flat: torch.Tensor) -> List[Tuple[nn.Module, _Part]]:
    """The trained layers and their places in the flat map; refuses what the pass could not give scores for."""
    place: Dict[int, torch.Tensor] = {}
    at = 0
    for p in model.parameters():
        place[id(p)] = flat[at:at + p.numel()].view(p.shape)
        at += p.numel()
    parts, owner = [], {}
    for name, m in model.named_modules():
        own = {n: p for n, p in m.named_parameters(recurse=False)}
        trained = {n: p for n, p in own.items() if p.requires_grad}
        for p in own.values():
            if id(p) in owner and p.requires_grad:
                _refuse("a parameter is shared by %s and %s" % (owner[id(p)], name))
            owner[id(p)] = name
        if not trained:
            continue
        if type(m) is nn.Linear:
            if "weight" not in trained:
                _refuse("the weight of %s is not trained, but its bias is" % name)
        elif type(m) is nn.LayerNorm:
            if len(m.normalized_shape) != 1:
                _refuse("%s normalises over %d dimensions" % (name, len(m.normalized_shape)))
        else:
            _refuse("%s (%s) has trained parameters: only those of linear layers and layer norms get scores; give the others requires_grad=False" %
                    (name, type(m).__name__))
        parts.append((m, _Part(name, place[id(m.weight)] if "weight" in trained else None,
                               place[id(m.bias)] if getattr(m, "bias", None) is not None and "bias" in trained else None)))
    if not parts:
        _refuse("the model has no trained linear layer or layer norm")
    return parts


_taken: set = set()              # layers of the passes under way, by id
_taking = threading.Lock()


@contextlib.contextmanager
def _layers_of(parts: List[Tuple[nn.Module, _Part]], state: _Pass):
    """The trained layers go by the functions above while this lasts: in this thread, others' calls are refused."""
    thread = threading.get_ident()

    def enter(part, x):
        if threading.get_ident() != thread:
            _refuse("layer %s is called by another thread than the one whose pass it is in" % part.name)
        state.enter(part, x.shape)

    def linear(m, part):
        def forward(x):
            enter(part, x)
            return _Linear.apply(x, m.weight, m.bias, part, state)
        return forward

    def norm(m, part):
        def forward(x):
            enter(part, x)
            return _LayerNorm.apply(x, m.weight, m.bias, m.eps, part, state)
        return forward

    layers = {id(m) for m, _ in parts}
    with _taking:
        for m, part in parts:
            if id(m) in _taken:
                _refuse("layer %s is in a pass already" % part.name)
            if "forward" in m.__dict__:
                _refuse("layer %s has a forward of its own, which the pass would leave out" % part.name)
        _taken.update(layers)
    try:
        for m, part in parts:
            m.forward = linear(m, part) if isinstance(m, nn.Linear) else norm(m, part)
        yield
    finally:
        for m, _ in parts:
            m.__dict__.pop("forward", None)
        with _taking:
            _taken.difference_update(layers)


def sensitivity_map(ctx: Ctx, model: nn.Module, batches: Iterable[Tuple[torch.Tensor, torch.Tensor]]) -> Sensitivity:
    """The map of a model over a client's samples.

    ``batches``: pairs of inputs, which ``model`` turns into logits [samples][tokens][vocabulary] (or [samples][vocabulary]), and int64
    targets of the logits' leading shape; a negative target is none (padding).  Every entry of the first dimension is a sample, in the
    layers too, and the model must not let one sample's activations depend on another's.  Scores are computed for the trained
    parameters of nn.Linear and nn.LayerNorm, each called once in a pass; a model that trains others, or uses these in another way (by a
    ``forward`` that was set on the module or under ``no_grad``, for instance), is refused.  Parameters without a score (those that are not trained,
    and those of layers that no gradient reaches) have 0, which he_select_mask takes last.  While a batch is passed through the model its trained layers' ``forward`` is replaced: calls by other threads are refused
    meanwhile, and so is a second pass.  Works under ``torch.autocast``.  No gradient is left behind, and the model's mode stays: with dropout, call
    ``model.eval()`` first.  Waits for the GPU at its end and reads the context's status, as he_ctx_status does: an error that the pass
    or a call before it left there is raised, and the status cleared."""
    params = list(model.parameters())
    if not params or not params[0].is_cuda:
        raise TypeError("expected a model on a CUDA device")
    flat = torch.zeros(sum(p.numel() for p in params), dtype=torch.float32, device=params[0].device)
    parts = _parts(model, flat)
    trained = [p for p in params if p.requires_grad]
    samples = rows = 0
    sums = torch.zeros(3, dtype=torch.float64, device=flat.device)
    for inputs, targets in batches:
        if targets.dim() == 0:
            _refuse("targets have no dimension of samples")
        count = targets.shape[0]
        if targets.numel() == 0:                             # a sample of no token has no gradient
            samples += count
            continue
        state = _Pass(ctx, count, flat.device)
        with _layers_of(parts, state), torch.enable_grad():
            logits = model(inputs)
            if logits.shape[:-1] != targets.shape:
                _refuse("targets of shape %s for logits of shape %s" % (tuple(targets.shape), tuple(logits.shape)))
            z, y = _rows(logits.detach()), targets.reshape(-1)
            logp, lse, entropy, _, _ = he_token_log_probs(ctx, z, y)
            dz = he_token_log_probs_backward(ctx, z, y, lse, torch.ones_like(lse))
            with torch.autocast(flat.device.type, enabled=False):        # each gradient is in the type of its part of the pass forward
                grads = torch.autograd.grad(logits, trained, dz.view(logits.shape), allow_unused=True)
            if any(g is not None for g in grads):
                _refuse("a parameter is used other than by its layer's call")
        counted = y >= 0
        sums += torch.stack([torch.where(counted, logp, 0).sum(dtype=torch.float64), entropy.sum(dtype=torch.float64), counted.sum()])
        samples += count
        rows += y.numel()
    if samples:
        flat /= samples
    log_prob, entropy, tokens = sums.tolist()
    status = he_ctx_status(ctx)
    if status != HE_OK:
        raise HeError(status, "sensitivity_map: the context's status")
    return Sensitivity(flat, samples, int(tokens), log_prob / max(1, tokens), entropy / max(1, rows))
