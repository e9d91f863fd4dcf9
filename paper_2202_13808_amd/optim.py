"""AdamW on the library's kernel: one pass over all parameters, states in 32 or in 8 bits.

The dropped cache shrinks what a training step keeps of its activations; the optimizer's states are the next largest
thing beside the weights.  ``AdamW(..., state_bits=8)`` keeps them in a quarter of their bytes, and bf16 parameters become
exact fp32 masters with 16 more bits each instead of an fp32 copy.  Clipping by the global norm costs one read of the
gradients: the factor goes from kernel to kernel on the device (``dropit_grad_norm``, ``dropit_adamw``).
"""
from __future__ import annotations

from typing import Any, Dict, List, Optional, Tuple

import torch

from . import layers

_DTYPES = (torch.float32, torch.bfloat16)
_GROUP_KEYS = ("lr", "betas", "eps", "weight_decay", "state_bits", "residual", "capturable")


def _memory_order(t: torch.Tensor) -> torch.Tensor:
    """A contiguous view of a dense tensor: its dimensions in the order in which they lie in memory."""
    if t.is_contiguous():
        return t
    order = sorted(range(t.dim()), key=lambda d: (t.stride(d), t.shape[d]), reverse=True)
    v = t.permute(order)
    if not v.is_contiguous():
        raise TypeError("AdamW takes dense parameters only, got shape %s with strides %s" % (tuple(t.shape), tuple(t.stride())))
    return v


def _same_layout(a: torch.Tensor, b: torch.Tensor) -> bool:
    return a.stride() == b.stride() or (a.is_contiguous() and b.is_contiguous())


def _contiguous(tensors: List[torch.Tensor]) -> bool:
    return layers._marshal().describe(tensors)[5]


def _all_in_memory_order(tensors: List[torch.Tensor]) -> List[torch.Tensor]:
    return tensors if _contiguous(tensors) else [_memory_order(t) for t in tensors]


class AdamW(torch.optim.Optimizer):
    """AdamW with decoupled weight decay over float32 and bfloat16 device parameters.  A group's parameters are on one device;
    with ``max_norm``, all groups' are.

    ``state_bits``  32 (fp32 moments) or 8 (blocks of 256 codes, see ``dropit_adamw``); a group may have its own
    ``residual``    bfloat16 parameters keep 16 more bits each and follow their fp32 values exactly (default); False rounds
                    them to bfloat16 every step, which loses updates of less than a 256th of a parameter
    ``max_norm``    the gradients' global 2-norm, over all groups, is clipped to this (None: not); ``last_grad_norm`` is then
                    the unclipped norm, a device scalar.  Copies of the optimizer keep both; ``state_dict()`` holds neither
    ``capturable``  the step count lives on the device, so that ``step()`` can be captured into a HIP graph and replayed.  All
                    parameters of a group then step together: a missing gradient is an error.  Take one step outside the
                    capture first (it makes the states).  ``lr`` and the other numbers are captured as they are.

    Moments, residuals and step counts are in ``state_dict()`` in their own types."""

    def __init__(self, params, lr: float = 1e-3, betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 1e-2, *, state_bits: int = 32, residual: bool = True,
                 max_norm: Optional[float] = None, capturable: bool = False) -> None:
        if max_norm is not None and not float(max_norm) > 0.0:
            raise ValueError("max_norm must be positive, got %r" % (max_norm,))
        self.max_norm = None if max_norm is None else float(max_norm)
        self.last_grad_norm: Optional[torch.Tensor] = None
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                                      residual=bool(residual), capturable=bool(capturable)))

    def __getstate__(self) -> Dict[str, Any]:
        # (copies and pickles carry what this says; torch's names the groups and the states only)
        return {**super().__getstate__(), "max_norm": self.max_norm, "last_grad_norm": self.last_grad_norm}

    def add_param_group(self, param_group: Dict[str, Any]) -> None:
        super().add_param_group(param_group)
        group = self.param_groups[-1]
        try:
            if isinstance(group["lr"], torch.Tensor):
                raise TypeError("lr must be a number")
            b1, b2 = group["betas"]
            if not (group["lr"] >= 0.0 and 0.0 <= b1 < 1.0 and 0.0 <= b2 < 1.0 and group["eps"] >= 0.0 and group["weight_decay"] >= 0.0):
                raise ValueError("lr, eps and weight_decay must not be negative, betas in [0, 1)")
            if group["state_bits"] not in (8, 32):
                raise ValueError("state_bits must be 8 or 32, got %r" % (group["state_bits"],))
            if len(set(map(id, group["params"]))) != len(group["params"]):
                raise ValueError("a parameter appears twice in a group")
            for p in group["params"]:
                if p.dtype not in _DTYPES:
                    raise TypeError("AdamW takes float32 and bfloat16 parameters, got %s" % p.dtype)
                _memory_order(p.detach())
        except Exception:
            self.param_groups.pop()
            raise

    # ---- states ----------------------------------------------------------------------------------
    def _new_state(self, p: torch.Tensor, group: Dict[str, Any], step: Any) -> Dict[str, Any]:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW's states are made by its first step: take one outside the capture")
        bits8 = group["state_bits"] == 8
        dtype = torch.uint8 if bits8 else torch.float32
        state: Dict[str, Any] = {"step": step, "exp_avg": torch.zeros_like(p, dtype=dtype, memory_format=torch.preserve_format),
                                 "exp_avg_sq": torch.zeros_like(p, dtype=dtype, memory_format=torch.preserve_format)}
        if bits8:
            blocks = (p.numel() + layers.ADAMW_BLOCK - 1) // layers.ADAMW_BLOCK
            for name in ("exp_avg_offset", "exp_avg_sq_offset"):
                state[name] = torch.zeros(blocks, dtype=torch.int16, device=p.device)
        if group["residual"] and p.dtype == torch.bfloat16:
            state["residual"] = torch.zeros_like(p, dtype=torch.int16, memory_format=torch.preserve_format)
        return state

    def moments(self, p: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """The moments of a parameter as values: fp32, or what the 8-bit codes stand for, in bfloat16."""
        state = self.state[p]
        if "exp_avg_offset" not in state:
            return state["exp_avg"], state["exp_avg_sq"]
        out = []
        for name, signed in (("exp_avg", True), ("exp_avg_sq", False)):
            values = torch.empty_like(state[name], dtype=torch.bfloat16)
            layers.adamw_unpack(_memory_order(state[name]), state[name + "_offset"], signed, values=_memory_order(values))
            out.append(values)
        return out[0], out[1]

    def load_state_dict(self, state_dict: Dict[str, Any]) -> None:
        """Loads what the pre-hooks make of ``state_dict``; the post-hooks find the states as they stay.  What does not fit the
        parameters (another optimizer's states, other types or sizes) is refused and changes nothing."""
        loaded: Dict[str, Any] = {}

        def behind_the_pre_hooks(_, sd: Dict[str, Any]) -> None:
            loaded.update(sd)
            for group in sd["param_groups"]:
                self._check_loaded_group(group)
            for p, group, state in self._states_of(loaded):
                self._check_loaded(p, group, state)
            for group in sd["param_groups"]:
                if group["capturable"] and len({int(sd["state"][i]["step"]) for i in group["params"] if sd["state"].get(i)}) > 1:
                    raise ValueError("the parameters of a capturable group must have made the same number of steps")

        def before_the_post_hooks(_) -> None:
            self._take_states(loaded)

        handles = (self.register_load_state_dict_pre_hook(behind_the_pre_hooks),
                   self.register_load_state_dict_post_hook(before_the_post_hooks, prepend=True))
        try:
            super().load_state_dict(state_dict)
        finally:
            for handle in handles:
                handle.remove()

    def _states_of(self, state_dict: Dict[str, Any]) -> List[Tuple[torch.Tensor, Dict[str, Any], Dict[str, Any]]]:
        """Parameter, saved group and saved state of every parameter."""
        saved = [(i, g) for g in state_dict["param_groups"] for i in g["params"]]
        own = [p for g in self.param_groups for p in g["params"]]
        return [(p, g, state_dict["state"].get(i, {})) for (i, g), p in zip(saved, own)]

    @staticmethod
    def _check_loaded_group(group: Dict[str, Any]) -> None:
        missing = [k for k in _GROUP_KEYS if k not in group]
        if missing:
            raise ValueError("not a group of this optimizer: it lacks %s (a load_state_dict pre-hook can turn another's states into its)"
                             % ", ".join(missing))
        if group["state_bits"] not in (8, 32):
            raise ValueError("state_bits must be 8 or 32, got %r" % (group["state_bits"],))

    @staticmethod
    def _check_loaded(p: torch.Tensor, group: Dict[str, Any], state: Dict[str, Any]) -> None:
        if not state:                                  # (no step yet)
            return
        bits8 = group["state_bits"] == 8
        moment = (torch.uint8 if bits8 else torch.float32, p.numel())
        kinds = {"exp_avg": moment, "exp_avg_sq": moment}
        if bits8:
            kinds["exp_avg_offset"] = kinds["exp_avg_sq_offset"] = (torch.int16, (p.numel() + layers.ADAMW_BLOCK - 1) // layers.ADAMW_BLOCK)
        if "residual" in state:
            if p.dtype != torch.bfloat16:
                raise ValueError("a state with a residual belongs to a bfloat16 parameter, not to one of %s" % p.dtype)
            kinds["residual"] = (torch.int16, p.numel())
        for name, (dtype, numel) in kinds.items():
            value = state.get(name)
            if not isinstance(value, torch.Tensor) or value.dtype != dtype or value.numel() != numel:
                raise ValueError("%s of a parameter of shape %s in %d-bit states must be %d elements of %s" % (
                    name, tuple(p.shape), group["state_bits"], numel, dtype))
        step = state.get("step", -1)
        step = step.item() if isinstance(step, torch.Tensor) and step.numel() == 1 else step
        if isinstance(step, torch.Tensor) or step != int(step) or step < 0:
            raise ValueError("a state's step must be a count, got %r" % (state.get("step"),))
        if bits8 and state["exp_avg"].shape == p.shape and not _same_layout(state["exp_avg"], p):
            raise ValueError("8-bit states go by the order of their parameter in memory: saved with strides %s, loaded with %s"
                             % (tuple(state["exp_avg"].stride()), tuple(p.stride())))

    def _take_states(self, state_dict: Dict[str, Any]) -> None:
        """The loaded states in their own types (torch's loading casts floating ones to their parameter's)."""
        counts: Dict[int, torch.Tensor] = {}           # a capturable group's parameters share one, which its step raises
        for p, group, state in self._states_of(state_dict):
            for name, value in state.items():
                if name == "step":
                    count: Any = int(value)
                    if group["capturable"]:
                        count = counts.setdefault(id(group), torch.full((1,), count, dtype=torch.int32, device=p.device))
                    self.state[p][name] = count
                elif not isinstance(value, torch.Tensor):
                    self.state[p][name] = value
                else:
                    own = torch.empty_like(p, dtype=value.dtype, memory_format=torch.preserve_format) if value.shape == p.shape \
                        else torch.empty(value.shape, dtype=value.dtype, device=p.device)
                    self.state[p][name] = own.copy_(value)
            if state and group["residual"] and p.dtype == torch.bfloat16 and "residual" not in state:
                # (saved of an fp32 parameter: the bf16 value as it is)
                self.state[p]["residual"] = torch.zeros_like(p, dtype=torch.int16, memory_format=torch.preserve_format)

    # ---- the step --------------------------------------------------------------------------------
    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        # of each launch: its group, the step count, parameters, gradients, states
        work: List[Tuple[Dict[str, Any], Any, List[torch.Tensor], List[torch.Tensor], List[Dict[str, Any]]]] = []
        for group in self.param_groups:
            pairs = [(p, p.grad) for p in group["params"]]
            params = [p for p, g in pairs if g is not None]
            if not params:
                continue
            grads = [g for _, g in pairs if g is not None]
            device = layers._marshal().describe(params)[4]
            if device == -1:
                raise RuntimeError("AdamW steps device parameters only: there is no CPU path")
            if device < 0:
                raise RuntimeError("the parameters of a group must be on one device: give each device a group of its own")
            if not (_contiguous(params) and _contiguous(grads)):
                grads = [self._grad(p, g) for p, g in zip(params, grads)]
            states = [self.state[p] for p in params]
            if group["capturable"]:
                if len(params) != len(group["params"]):
                    raise RuntimeError("a capturable group steps together: %d of its %d parameters have no gradient"
                                       % (len(group["params"]) - len(params), len(group["params"])))
                count = next((s["step"] for s in states if s), 0)
                if not isinstance(count, torch.Tensor):        # (a new group, or one that was not capturable before)
                    if any(s and s["step"] != count for s in states):
                        raise RuntimeError("the parameters of a capturable group must have made the same number of steps")
                    if torch.cuda.is_current_stream_capturing():
                        raise RuntimeError("AdamW's states are made by its first step: take one outside the capture")
                    count = torch.full((1,), count, dtype=torch.int32, device=params[0].device)
                    for s in states:
                        if s:
                            s["step"] = count
                for p, s in zip(params, states):
                    if not s:
                        s.update(self._new_state(p, group, count))
                self._check_layouts(params, states)
                work.append((group, count, params, grads, states))
                continue
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("capturing AdamW.step() needs capturable=True: a replay would repeat one step's count")
            for p, s in zip(params, states):
                if not s:
                    s.update(self._new_state(p, group, 0))
                elif isinstance(s["step"], torch.Tensor):      # (the group was capturable before)
                    s["step"] = int(s["step"].item())
            self._check_layouts(params, states)
            counts = [s["step"] for s in states]
            for t in sorted(set(counts)):
                at = [j for j, c in enumerate(counts) if c == t]
                whole = len(at) == len(counts)
                pick = lambda x: x if whole else [x[j] for j in at]  # noqa: E731
                work.append((group, t + 1, pick(params), pick(grads), pick(states)))
        if not work:
            return loss
        scale = None
        if self.max_norm is not None:
            both = layers.grad_norm(_all_in_memory_order([g for w in work for g in w[3]]), max_norm=self.max_norm)
            self.last_grad_norm, scale = both[0], both[1:]
        for group, t, params, grads, states in work:
            if isinstance(t, torch.Tensor):
                t.add_(1)
            else:
                for s in states:
                    s["step"] = t
            types = [p.dtype for p in params]
            for dtype in _DTYPES:
                at = [j for j, d in enumerate(types) if d == dtype]
                if at:
                    whole = len(at) == len(types)
                    pick = lambda x: x if whole else [x[j] for j in at]  # noqa: E731
                    self._launch(group, t, pick(params), pick(grads), pick(states), scale)
        return loss

    @staticmethod
    def _check_layouts(params, states) -> None:
        """Moments and residuals go by their parameter's order in memory; all of a state are made alike."""
        own = [s["exp_avg"] for s in states]
        if not (_contiguous(params) and _contiguous(own)) and not all(map(_same_layout, own, params)):
            raise RuntimeError("a parameter's strides have changed since its states were made")

    @staticmethod
    def _grad(p: torch.Tensor, g: torch.Tensor) -> torch.Tensor:
        if g.stride() != p.stride() and not (g.is_contiguous() and p.is_contiguous()):
            g = torch.empty_like(p, dtype=g.dtype, memory_format=torch.preserve_format).copy_(g)
        return g

    def _launch(self, group: Dict[str, Any], t: Any, params, grads, states, scale) -> None:
        column = lambda name: _all_in_memory_order([s[name] for s in states])  # noqa: E731
        more = {}
        if group["state_bits"] == 8:
            more = {"m_offset": [s["exp_avg_offset"] for s in states], "v_offset": [s["exp_avg_sq_offset"] for s in states]}
        if "residual" in states[0]:
            more["residual"] = column("residual")
        layers.adamw(_all_in_memory_order(params), _all_in_memory_order(grads), column("exp_avg"), column("exp_avg_sq"), lr=group["lr"],
                     betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"], step=t, grad_scale=scale, **more)
        torch.autograd.graph.increment_version(params)  # (a graph that saved them must not go backward with the new values)
