"""AdamW over every tensor of a network at once, with moments in 32 or in 8 bits.

A network of wavelet convolutions has many small tensors (a kernel and a scale
for each level and layer). One step takes one launch for every 88 of them; the
moments of a parameter group lie in two buffers, one after the other.
"""
import torch

from . import autograd, binding

_M32 = 0xFFFFFFFF
_DTYPES = (torch.float32, torch.bfloat16, torch.float16)


def _mix(x):
    x = ((x ^ (x >> 15)) * 0x85EBCA6B) & _M32
    x = ((x ^ (x >> 13)) * 0xC2B2AE35) & _M32
    return x ^ (x >> 16)


def rounding_key(seed, step, group):
    """The key of the random bits that round one group's 8-bit moments in one step."""
    a = _mix((seed * 0x9E3779B1 + step * 0x9E3779B9) & _M32)
    return _mix((group * 0x9E3779B1 + a) & _M32)


def _strides_fill(t):
    """Whether the tensor's elements fill one run of memory, in any order of its dimensions."""
    run = 1
    for stride, n in sorted((stride, n) for n, stride in zip(t.shape, t.stride()) if n != 1):
        if stride != run:
            return t.numel() == 0
        run *= n
    return True


def _order(t):
    """The order of a dense tensor's memory: () for that of its shape, else its strides (0 for a dimension of one
    element, whose stride says nothing)."""
    return () if t.is_contiguous() else tuple(stride if n > 1 else 0 for n, stride in zip(t.shape, t.stride()))


class AdamW(torch.optim.Optimizer):
    """AdamW (decoupled weight decay) on GPU parameters in float32, bfloat16 or float16:

        m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
        p = p (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)

    computed in float32 and rounded to the parameter's type once. With `state_bits` = 32 the moments are float32. With
    8 they take one byte an element and one for every 64 elements, as small floats under a shared power of two; they
    are rounded at random, by bits that depend on `seed`, the step and the element alone, so that a step that is
    repeated gives the same bits. What is below about 2^-16 of its block's largest gradient keeps no size of its own in
    them: its updates are those of a gradient of about that size, or smaller. A block of 64 that meets a value that is
    not finite stands for NaN from then on, as a 32-bit moment does.

    The moments are allocated with the group, in the order of the parameters' memory. `state[p]` holds views of them:
    "exp_avg" and "exp_avg_sq" (shaped as p with 32 bits; the codes, one an element in the order of memory, with 8),
    "exp_avg_scale", "exp_avg_sq_scale" and "order" (8 bits: which order that is, () or the strides), and "step", the
    number of steps p has taken; they are changed by writing into the views. A parameter without a gradient is left
    alone; a group's list of parameters stays as it was added. Where a parameter's memory gets another order (to
    channels_last, say), moments in 32 bits follow it; those in 8 bits share their scales in the old order, so that a
    step is refused unless it is the first.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=32, seed=0):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits must be 8 or 32, got {state_bits}")
        self.state_bits, self.seed = state_bits, int(seed)
        self._buffers = []  # of each group: exp_avg, exp_avg_sq, their scales (8 bits), step, params, offsets, numel, orders
        self._native = []   # the same for the native host path
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        return {**super().__getstate__(), "state_bits": self.state_bits, "seed": self.seed}

    def __setstate__(self, state):
        """A copy: its groups' buffers are allocated anew and take the moments and steps over."""
        super().__setstate__(state)
        self._buffers, self._native = [], []
        for group in self.param_groups:
            held = [self.state[p] for p in group["params"]]
            self._allocate(group)
            buffers = self._buffers[-1]
            for i, (p, old) in enumerate(zip(group["params"], held)):
                for k, t in self.state[p].items():
                    if k == "order":  # (not p's, where that changed since the last step)
                        self.state[p][k] = buffers["orders"][i] = old[k]
                    else:
                        t.copy_(old[k])
            self._native[-1] = self._plan(group["params"], buffers)

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        group = self.param_groups[-1]
        try:
            self._check_group(group)
            self._allocate(group)
        except BaseException:  # (an argument, or no memory for the moments)
            self.param_groups.pop()
            del self._buffers[len(self.param_groups):], self._native[len(self.param_groups):]
            for p in group["params"]:
                self.state.pop(p, None)
            raise

    def _check_group(self, group):
        _hyperparameters(group)
        devices = {p.device for g in self.param_groups for p in g["params"]}
        for p in group["params"]:
            if not p.is_cuda:
                raise ValueError("AdamW steps GPU tensors only")
            if p.dtype not in _DTYPES:
                raise ValueError(f"parameters must be float32, bfloat16 or float16, got {p.dtype}")
            if p.layout != torch.strided or not _strides_fill(p):
                raise ValueError(f"a parameter of shape {tuple(p.shape)} and strides {p.stride()} does not fill its "
                                 "memory")
        if len(devices) > 1:
            raise ValueError(f"all parameters must be on one device, got {sorted(map(str, devices))}")

    def _allocate(self, group):
        block, params, offsets, end = binding.ADAMW_BLOCK, group["params"], [], 0
        for p in params:
            offsets.append(end)
            end += -(-p.numel() // block) * block
        coded = self.state_bits == 8
        new = lambda n: torch.zeros(n, dtype=torch.uint8 if coded else torch.float32,  # noqa: E731
                                    device=params[0].device if params else "cpu")
        buffers = {"exp_avg": new(end), "exp_avg_sq": new(end)}
        if coded:
            buffers.update(exp_avg_scale=new(end // block), exp_avg_sq_scale=new(end // block))
        buffers.update(step=torch.zeros(len(params), dtype=torch.int64), params=list(params), offsets=offsets,
                       numel=[p.numel() for p in params], orders=[_order(p) for p in params])
        self._buffers.append(buffers)
        self._native.append(self._plan(params, buffers))
        for i, p in enumerate(params):
            self._show(buffers, i, p)

    def _plan(self, params, buffers):
        """The group for the native host path; None without it, and for no parameters."""
        ext = autograd.load_block(params[0]) if params else False
        return ext.AdamWGroup(*(buffers[n] for n in ("params", "offsets", "numel", "orders", "step", "exp_avg",
                                                      "exp_avg_sq")),
                              *(buffers.get(n) for n in ("exp_avg_scale", "exp_avg_sq_scale"))) if ext else None

    def _show(self, buffers, i, p):
        """state[p] as views of the group's buffers, in the present order of p's memory."""
        block, at, n = binding.ADAMW_BLOCK, buffers["offsets"][i], p.numel()
        buffers["orders"][i] = _order(p)
        self.state[p] = state = {"step": buffers["step"][i]}
        for name in ("exp_avg", "exp_avg_sq"):
            if self.state_bits == 8:
                state[name] = buffers[name][at:at + n]
                state[name + "_scale"] = buffers[name + "_scale"][at // block:at // block - (-n // block)]
                state["order"] = buffers["orders"][i]
            else:
                state[name] = buffers[name][at:at + n].as_strided(p.shape, p.stride())

    def _reorder(self, index, i, p):
        """Bring the moments of a parameter whose memory has another order than they have into that order."""
        buffers, held = self._buffers[index], self.state[p]
        if self.state_bits == 32 and held["exp_avg"].shape == p.shape:
            held = {name: held[name].clone() for name in ("exp_avg", "exp_avg_sq")}
        elif int(held["step"]):
            raise ValueError(f"a parameter of shape {tuple(p.shape)} changed its order of memory: its moments are in "
                             "the old one")
        else:  # there are none yet
            held = {}
        self._show(buffers, i, p)
        for name, moment in held.items():
            self.state[p][name].copy_(moment)
        self._native[index] = self._plan(self.param_groups[index]["params"], buffers)

    def step(self, closure=None, grad_scale=None):
        """One step. grad_scale: a float32 GPU tensor of one element that every gradient is multiplied with (to undo
        a loss scale, or to clip), or None."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if not any(g["params"] for g in self.param_groups):
            return loss
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("an AdamW step cannot be captured: the bias corrections of its step would be replayed")
        ext = autograd._block
        if not (ext and all(native or not g["params"] for native, g in zip(self._native, self.param_groups)) and
                ext.adamw_step(self._native, [g["params"] for g in self.param_groups],
                               [_hyperparameters(g) for g in self.param_groups], self.state_bits, self.seed & _M32,
                               grad_scale)):
            self._step(grad_scale)
        return loss

    @torch.no_grad()
    def _step(self, grad_scale):
        device, taken, calls = None, [], {}  # calls: by the parameters' type, (groups, tensors)
        for index, (group, buffers) in enumerate(zip(self.param_groups, self._buffers)):
            lr, beta1, beta2, eps, decay = _hyperparameters(group)
            if len(group["params"]) != len(buffers["params"]) or \
                    any(p is not q for p, q in zip(group["params"], buffers["params"])):
                raise ValueError(f"the parameters of group {index} are not those it was added with: add a group instead")
            places = {}  # of (type, step) in the call's groups
            steps = buffers["step"].tolist()
            for i, p in enumerate(group["params"]):
                if p.grad is None:
                    continue
                grad = _gradient(p, buffers, i)
                if _order(p) != buffers["orders"][i]:
                    self._reorder(index, i, p)
                device, step = p.device, steps[i] + 1
                taken.append((buffers["step"], i, p, grad))  # a gradient that was copied lives until the launch
                if not p.numel():  # (a group of nothing else has no buffers)
                    continue
                code = binding._dtype_code(p)
                groups, tensors = calls.setdefault(code, ([], []))
                if (code, step) not in places:
                    places[code, step] = len(groups)
                    scales = [buffers[n].data_ptr() if n in buffers else None
                              for n in ("exp_avg_scale", "exp_avg_sq_scale")]
                    groups.append(binding.AdamWGroup(lr, beta1, beta2, eps, decay, step,
                                                     rounding_key(self.seed, step, index),
                                                     buffers["exp_avg"].data_ptr(), buffers["exp_avg_sq"].data_ptr(),
                                                     *scales))
                tensors.append(binding.AdamWTensor(p.data_ptr(), grad.data_ptr(), p.numel(), buffers["offsets"][i],
                                                   places[code, step]))
        if device is None:
            return
        if grad_scale is not None:
            binding._require(grad_scale, "grad_scale", torch.float32, device=device)
            if grad_scale.numel() != 1:
                raise ValueError(f"grad_scale must have one element, got shape {tuple(grad_scale.shape)}")
        stream = binding._stream(device)
        with binding._on(device):
            for code, (groups, tensors) in calls.items():
                binding._check(binding.wtconv_adamw_step(groups, tensors, code, self.state_bits,
                                                         binding._ptr(grad_scale), stream))
        for steps, i, _, _ in taken:
            steps[i] += 1
        torch.autograd.graph.increment_version([p for _, _, p, _ in taken])

    def moments(self, dtype=torch.bfloat16):
        """(exp_avg, exp_avg_sq) of each group, every parameter's from its first element's place on (a multiple of
        64). With 32 bits these are the buffers themselves; with 8 bits the values that the codes stand for, as new
        tensors of `dtype` (bfloat16 holds each exactly down to 2^-126)."""
        if self.state_bits == 32:
            return [(b["exp_avg"], b["exp_avg_sq"]) for b in self._buffers]
        if dtype not in _DTYPES:
            raise ValueError(f"the moments' values are float32, bfloat16 or float16, not {dtype}")
        ext = autograd._block
        return [ext and native and ext.adamw_moments(native, dtype) or
                binding.adamw_moments(b["exp_avg"], b["exp_avg_scale"], b["exp_avg_sq"], b["exp_avg_sq_scale"], dtype)
                if b["params"] else (b["exp_avg"].to(dtype), b["exp_avg_sq"].to(dtype))
                for b, native in zip(self._buffers, self._native)]

    def state_dict(self):
        """The moments and hyperparameters as torch's optimizers give them, and the seed."""
        return {**super().state_dict(), "seed": self.seed}

    def load_state_dict(self, state_dict):
        """Copy the hyperparameters, the moments and the seed (if it is there) of a state_dict() of an optimizer with
        the same groups, shapes and state_bits into this one."""
        for hook in self._optimizer_load_state_dict_pre_hooks.values():
            changed = hook(self, state_dict)
            state_dict = state_dict if changed is None else changed
        saved, groups = state_dict["state"], state_dict["param_groups"]
        if [len(g["params"]) for g in groups] != [len(g["params"]) for g in self.param_groups]:
            raise ValueError("the state has other parameter groups")
        places = [(index, i, p, saved[j]) for index, (ours, g) in enumerate(zip(self.param_groups, groups))
                  for i, (p, j) in enumerate(zip(ours["params"], g["params"])) if j in saved]
        for _, _, p, state in places:
            # (a state without "order" is a dense parameter's)
            ours, state = {**self.state[p]}, {**state}
            if tuple(state.pop("order", ())) != (_order(p) if ours.pop("order", None) is not None else ()):
                raise ValueError(f"the 8-bit state is of a parameter in another order of memory than this one of shape "
                                 f"{tuple(p.shape)}")
            if set(state) != set(ours) or any(state[k].shape != ours[k].shape or state[k].dtype != ours[k].dtype
                                              for k in ours):
                raise ValueError("the state is not of these parameters, or was held in other bits")
        for index, i, p, state in places:
            buffers = self._buffers[index]
            if _order(p) != buffers["orders"][i]:
                self._show(buffers, i, p)
                self._native[index] = self._plan(self.param_groups[index]["params"], buffers)
            for k, t in self.state[p].items():
                if k != "order":
                    t.copy_(state[k])
        for ours, g in zip(self.param_groups, groups):
            ours.update({k: v for k, v in g.items() if k != "params"})
        self.seed = int(state_dict.get("seed", self.seed))
        for hook in self._optimizer_load_state_dict_post_hooks.values():
            hook(self)


def _gradient(p, buffers, i):
    """The gradient of the group's parameter i, in the order of its memory."""
    grad = p.grad
    if grad.layout != torch.strided:
        raise ValueError("AdamW takes dense gradients only")
    if p.numel() != buffers["numel"][i] or p.dtype not in _DTYPES or p.device != buffers["exp_avg"].device or \
            not _strides_fill(p):
        raise ValueError(f"a parameter of shape {tuple(p.shape)} changed its size, type or device, or does not fill its "
                         "memory any more")
    if grad.dtype != p.dtype or grad.device != p.device:
        raise ValueError(f"a gradient is {grad.dtype} on {grad.device}, its parameter {p.dtype} on {p.device}")
    if grad.stride() != p.stride() or not _strides_fill(grad):
        grad = torch.empty_like(p, requires_grad=False).copy_(grad)
    return grad


def _hyperparameters(group):
    """(lr, beta1, beta2, eps, weight_decay) of a group as numbers, checked."""
    lr, (beta1, beta2), eps, decay = float(group["lr"]), group["betas"], group["eps"], group["weight_decay"]
    for name, v in (("lr", lr), ("eps", eps), ("weight_decay", decay)):
        if not 0 <= v < float("inf"):
            raise ValueError(f"{name} must be a number >= 0, got {v}")
    for v in (beta1, beta2):
        if not 0 <= v < 1:
            raise ValueError(f"betas must be in [0, 1), got {group['betas']}")
    return lr, float(beta1), float(beta2), float(eps), float(decay)
