"""AdamW over the parameters of a model, one launch for every 56 of them (clear_block_adamw).

    from paper_2412_16112_amd.optim import AdamW
    opt = AdamW(model.parameters(), lr=1e-4, weight_decay=0.01, state_bits=8)
    loss.backward(); opt.step(); opt.zero_grad()

The optimizer owns the states, and the fp32 masters if asked for (for bf16 parameters: small steps are not lost in the rounding).  Where tensors lie
is written down once; a step hands over the gradients.  One set of numbers (lr, ...) holds for all parameters: those that are to have others, norms and biases without decay, say,
go to an optimizer of their own."""
import torch

from . import clear_attn as ca
from . import clear_block as cb


class AdamW:
    def __init__(self, params, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, state_bits=32, masters=False):
        self.params = list(params)
        if state_bits not in (8, 32):
            raise ca.ClearAttnError(ca.CLEAR_ERR_INVALID_ARG, "state_bits must be 32 or 8")
        self.hyper = dict(lr=lr, beta1=beta1, beta2=beta2, eps=eps, weight_decay=weight_decay)
        self.grad_norm = None  # of the last step that was given a bound for it
        self.state_bits = state_bits
        states = [cb.adamw_state(p.detach(), state_bits) for p in self.params]
        # (tuples, and properties without a setter: a step works on these tensors, others in their place would be ignored)
        self._masters = tuple(p.detach().float().clone() for p in self.params) if masters else None
        self._exp_avgs, self._exp_avg_sqs = tuple(s[0] for s in states), tuple(s[1] for s in states)
        self._scales = tuple(s[2] for s in states) if state_bits == 8 else None
        # one table of descriptors for each (device, dtype), with the number of updates that each of its parameters has had
        self._tables = []
        places = {}
        for i, p in enumerate(self.params):
            places.setdefault((p.device, p.dtype), []).append(i)
        for members in places.values():
            of = lambda kept: None if kept is None else [kept[i] for i in members]
            params = [self.params[i].detach() for i in members]
            ca._dtype_code(params[0])
            table = cb._table(params, of(self.exp_avgs), of(self.exp_avg_sqs), of(self.masters), of(self.scales))
            self._tables.append((members, params, table, [0] * len(members), of(self.masters)))

        spans = sorted((p.device.index, p.data_ptr(), p.data_ptr() + p.numel() * p.element_size()) for p in self.params if p.numel())
        if any(a[0] == b[0] and b[1] < a[2] for a, b in zip(spans, spans[1:])):
            raise ca.ClearAttnError(ca.CLEAR_ERR_INVALID_ARG, "parameters share memory")

    exp_avgs = property(lambda self: self._exp_avgs)
    exp_avg_sqs = property(lambda self: self._exp_avg_sqs)
    scales = property(lambda self: self._scales)
    masters = property(lambda self: self._masters)

    @property
    def steps(self):
        """The updates of the parameter that has had most of them.  Set, it holds for all."""
        return max((max(counts) for _, _, _, counts, _ in self._tables), default=0)

    @steps.setter
    def steps(self, n):
        for _, _, _, counts, _ in self._tables:
            counts[:] = [n] * len(counts)

    def step(self, grads=None, grad_scale=None, stream=None, max_norm=None, **hyper):
        """One step with the parameters' .grad, or with `grads` (a list in their order); entries that are None are skipped: a parameter counts its own updates.  Keyword arguments
        (lr, ...) hold for this step only.  grad_scale: an fp32 device scalar that the gradients are multiplied by.  max_norm: with it, the gradients are scaled down to that norm of all of
        them together (times grad_scale) where they have a larger one; `grad_norm` then is what they had, an fp32 scalar on the device (0 where there is no gradient).  The gradients themselves stay as they are."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if len(grads) != len(self.params):
            raise ca.ClearAttnError(ca.CLEAR_ERR_MISMATCH, "one gradient for each parameter")
        h = dict(self.hyper, **hyper)
        given = []
        for members, params, table, _, _ in self._tables:  # (everything is checked before anything is updated; the numbers, which are everybody's, with the first launch)
            if any(self.params[i].data_ptr() != p.data_ptr() for i, p in zip(members, params)):
                raise ca.ClearAttnError(ca.CLEAR_ERR_MISMATCH, "a parameter has moved since the optimizer was made")
            cb._check_scale(grad_scale, params[0].device)
            given.append(cb._set_grads(table, params, [grads[i] for i in members]))
        norm = self.grad_norm
        if max_norm is not None:
            if any(g is not None for g in grads):
                norm, grad_scale = cb.grad_norm(grads, max_norm=max_norm, grad_scale=grad_scale, stream=stream)
            else:
                norm = torch.zeros((), dtype=torch.float32, device=self.params[0].device) if self.params else None
        for (_, params, table, counts, masters), some in zip(self._tables, given):
            for n in sorted(set(counts)):  # (parameters that have had as many updates go together: all of them, unless gradients were missing; those without one are skipped)
                rows = table if counts.count(n) == len(counts) else table[[c == n for c in counts]]
                cb._launch(rows, params[0], self.state_bits == 8, n + 1, h["lr"], h["beta1"], h["beta2"], h["eps"], h["weight_decay"], grad_scale, stream)
            counts[:] = [c + 1 for c in counts] if some is None else [c + (i in some) for i, c in enumerate(counts)]
            cb._updated(some, params, masters)
        self.grad_norm = norm  # (not of a step that was refused)

    def state_dict(self):
        """What load_state_dict takes: the states themselves (not copies), the masters, each parameter's number of updates and the numbers of a step."""
        updates = [0] * len(self.params)
        for members, _, _, counts, _ in self._tables:
            for i, n in zip(members, counts):
                updates[i] = n
        lists = {name: None if kept is None else list(kept) for name, kept in self._kept()}
        return dict(lists, state_bits=self.state_bits, updates=updates, hyper=dict(self.hyper))

    def load_state_dict(self, state):
        """Copies another optimizer's state into this one's tensors: of as many parameters of the same shapes, in their order, with states of as many bits, and masters if this one
        has them.  With masters the next step starts from these, whatever the parameters hold."""
        refuse = lambda what: cb._refuse("the state does not fit: " + what, ca.CLEAR_ERR_MISMATCH)
        missing = {"state_bits", "updates", "hyper", *dict(self._kept())} - set(state)
        if missing:
            refuse("%s missing" % ", ".join(sorted(missing)))
        if state["state_bits"] != self.state_bits:
            refuse("states of %s bits" % state["state_bits"])
        if len(state["updates"]) != len(self.params) or any(n < 0 for n in state["updates"]):
            refuse("a number of updates for each parameter is needed")
        copies = []
        for name, kept in self._kept():
            if (kept is None) != (state[name] is None) or (kept is not None and len(kept) != len(state[name])):
                refuse(name)
            for to, given in zip(kept or (), state[name] or ()):
                pairs = list(zip(to, given)) if name == "scales" else [(to, given)]
                if name == "scales" and len(given) != 2:
                    refuse(name)
                for a, b in pairs:
                    if a.shape != b.shape or a.dtype != b.dtype:
                        refuse("%s of another shape or type" % name)
                    copies.append((a, b))
        for a, b in copies:
            a.copy_(b)
        for members, _, _, counts, _ in self._tables:
            counts[:] = [state["updates"][i] for i in members]
        self.hyper = dict(state["hyper"])

    def _kept(self):
        return (("exp_avgs", self._exp_avgs), ("exp_avg_sqs", self._exp_avg_sqs), ("scales", self._scales), ("masters", self._masters))

    def zero_grad(self):
        for p in self.params:
            p.grad = None
