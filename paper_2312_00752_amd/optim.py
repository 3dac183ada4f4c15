"""AdamW on the library's kernel (include/ss_adamw.h): all tensors of a group in a launch, moments in float32 or in 8 bits."""
import torch

from . import binding as B


class AdamW(torch.optim.Optimizer):
    """AdamW with decoupled weight decay over GPU tensors in float32 or bfloat16.

    ``state_bits`` 8 holds the moments in a byte each and a scale for every 256 elements.  Tensors in bfloat16 get a float32 copy that is
    updated in their place (``master=False``: none, the sum is rounded to bfloat16).  What is written to such a parameter from outside (a model
    loaded after its optimiser was made, a clamp, averaged weights) is taken into the copy by the next step, for the elements that no longer are the copy's
    rounding; a write that torch counts no version for (through ``.data``) or that comes between a graph's replays needs a call of
    ``refresh_masters``.  All state is allocated here, and steps are counted on the device, once for
    a group, so a step can be captured in a graph and replayed.  A tensor without a gradient is left out of a step, though its group's count goes on.
    A group's ``lr`` may be a float32 tensor of one element on the GPU, which a graph reads as it is at its replay."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=32, master=True):
        self._seen = {}   # parameters with a master: their version and memory when the two last agreed
        super().__init__(params, {"lr": lr, "betas": betas, "eps": eps, "weight_decay": weight_decay, "state_bits": state_bits, "master": master})

    def add_param_group(self, group):
        super().add_param_group(group)
        group = self.param_groups[-1]
        refused = None
        if group["state_bits"] not in (8, 32):
            refused = "state_bits must be 8 or 32, got %r" % (group["state_bits"],)
        elif any(p.dtype not in (torch.float32, torch.bfloat16) or not p.is_cuda or not p.is_contiguous() for p in group["params"]):
            refused = "parameters must be contiguous float32 or bfloat16 tensors on the GPU"
        if refused:
            self.param_groups.pop()
            raise ValueError(refused)
        for p in group["params"]:
            s = self.state[p]
            eight = group["state_bits"] == 8
            s["m"] = torch.zeros(p.shape, dtype=torch.int8 if eight else torch.float32, device=p.device)
            s["v"] = torch.zeros(p.shape, dtype=torch.uint8 if eight else torch.float32, device=p.device)
            if eight:
                blocks = -(-p.numel() // B.SS_ADAMW_BLOCK)
                s["m_scale"], s["v_scale"] = (torch.zeros(blocks, dtype=torch.float32, device=p.device) for _ in range(2))
            if p.dtype == torch.bfloat16 and group["master"]:
                s["master"] = p.detach().float()
        self._agree(group["params"])
        device = group["params"][0].device if group["params"] else "cuda"
        group["count"] = torch.zeros(2, dtype=torch.int32, device=device)

    def __setstate__(self, state):   # of a copy or a pickle, whose parameters are other tensors
        super().__setstate__(state)
        self._seen = {}

    def _agree(self, params):
        for p in params:
            if "master" in self.state[p]:
                self._seen[p] = p._version, p.data_ptr()

    def _follow(self, params, every=False):
        """Masters of parameters that have been written since they agreed (or of all) take the elements that are not their rounding.  Returns the parameters whose masters agree
        from here on: what a capture records has not happened yet."""
        late = [p for p in params if "master" in self.state[p] and (every or self._seen.get(p) != (p._version, p.data_ptr()))]
        for p in late:
            master = self.state[p]["master"]
            master.copy_(torch.where(p == master.to(p.dtype), master, p.float()))
        if not late or not torch.cuda.is_current_stream_capturing():
            return params
        for p in late:
            self._seen.pop(p, None)
        return [p for p in params if p in self._seen]

    @torch.no_grad()
    def refresh_masters(self):
        """Takes what was written to bfloat16 parameters into their float32 copies.  A step does it by itself but for writes that torch does not count and
        steps of a graph; called before a capture it keeps the graph free of it where there was a write or a loaded state."""
        for group in self.param_groups:
            self._agree(self._follow(group["params"], every=True))

    @torch.no_grad()
    def step(self, closure=None, grad_scale=None):
        """``grad_scale``: a float32 tensor of one element that the gradients are multiplied with (of clipping, or of a scaled loss)."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            params = [p for p in group["params"] if p.grad is not None]
            agreeing = self._follow(params)
            states = [self.state[p] for p in params]
            each = lambda name: [s.get(name) for s in states]
            eight = group["state_bits"] == 8
            B.ss_adamw_step(params, [p.grad.contiguous() for p in params], each("m"), each("v"), group["count"], group["lr"],
                            betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"], master=each("master"),
                            m_scale=each("m_scale") if eight else None, v_scale=each("v_scale") if eight else None, grad_scale=grad_scale)
            torch.autograd.graph.increment_version(params)   # a graph that still needs them as they were is told
            self._agree(agreeing)
        return loss

    @torch.no_grad()
    def load_state_dict(self, state):
        """Of an optimiser of the same groups.  What is loaded is copied into this one's tensors, which a captured step goes on using.  The parameters may be loaded before or
        behind it; where they are not the loaded masters' rounding, the parameters count."""
        groups = state["param_groups"]
        if [len(g["params"]) for g in groups] != [len(g["params"]) for g in self.param_groups]:
            raise ValueError("the loaded state has other parameter groups")
        for theirs, mine in zip(groups, self.param_groups):
            if (theirs["state_bits"], theirs["master"]) != (mine["state_bits"], mine["master"]):
                raise ValueError("the loaded state is of state_bits %r and master %r" % (theirs["state_bits"], theirs["master"]))
            for k, p in zip(theirs["params"], mine["params"]):
                given, own = state["state"][k], self.state[p]
                if {n: (t.dtype, t.shape) for n, t in given.items()} != {n: (t.dtype, t.shape) for n, t in own.items()}:
                    raise ValueError("the loaded state is of other tensors")
        for theirs, mine in zip(groups, self.param_groups):
            for k, p in zip(theirs["params"], mine["params"]):
                for name, t in self.state[p].items():
                    t.copy_(state["state"][k][name])
                self._seen.pop(p, None)
            mine["count"].copy_(theirs["count"])
            for name, value in theirs.items():
                if name not in ("params", "count"):
                    if name == "lr" and isinstance(mine["lr"], torch.Tensor):
                        mine["lr"].fill_(float(value))
                    elif isinstance(value, torch.Tensor):   # read onto whichever device
                        mine[name] = value.to(mine["count"].device, torch.float32 if name == "lr" else value.dtype, copy=True)
                    else:
                        mine[name] = value
