"""Buffers of an AdamW update over many tensors: the moments, and the device table that names the tensors.  The update itself is one launch of
the library."""
import torch

from . import binding as B


class AdamW:
    """Decoupled weight decay over a list of tensors, moments in 32 or in 8 bits.

    weights: fp32; grads: fp32 or bf16, all of one type, of the same sizes; lowp: bf16 copies of the weights (a list with None where there is none), or
    None.  weight_decay and lr_scale: one value for each tensor, or one for all.  The tensors have to be contiguous and stay where they are: the
    table holds their addresses.  state: the moments of an earlier run, {"m": [...], "v": [...], "exps": [...]} as state_dict() gives them; zeros
    otherwise.  8-bit moments (uint8, with two exponents for every 256 elements) take 2 bytes a parameter in place of 8."""

    def __init__(self, weights, grads, lowp=None, weight_decay=0.0, lr_scale=1.0, state_bits=32, state=None):
        n = len(weights)
        lowp = [None] * n if lowp is None else list(lowp)
        each = lambda v: [float(v)] * n if not hasattr(v, "__len__") else [float(x) for x in v]   # noqa: E731
        self.weight_decay, self.lr_scale = each(weight_decay), each(lr_scale)
        if not n or any(len(t) != n for t in (grads, lowp, self.weight_decay, self.lr_scale)):
            raise ValueError("AdamW: one gradient, copy, weight decay and lr scale for each of the weights")
        for w, g, p in zip(weights, grads, lowp):
            if w.dtype is not torch.float32 or g.dtype is not grads[0].dtype or (p is not None and p.dtype is not torch.bfloat16):
                raise TypeError("AdamW: weights are fp32, gradients of one type, copies bf16")
            if w.numel() != g.numel() or (p is not None and p.numel() != w.numel()) or not all(t is None or t.is_contiguous() for t in (w, g, p)):
                raise ValueError("AdamW: a weight, its gradient and its copy are contiguous and of one size")
        if state_bits not in (8, 32):
            raise ValueError("AdamW: moments in 8 or in 32 bits")
        self.weights, self.grads, self.lowp, self.state_bits = list(weights), list(grads), lowp, state_bits
        kind = torch.uint8 if state_bits == 8 else torch.float32
        blocks = [-(-w.numel() // B.ADAMW_BLOCK) for w in weights]
        if state is None:
            state = {k: [torch.zeros(w.numel(), dtype=kind, device=w.device) for w in weights] for k in ("m", "v")}
            if state_bits == 8:
                state["exps"] = [torch.zeros(b, 2, dtype=torch.uint8, device=w.device) for b, w in zip(blocks, weights)]
        self.m, self.v, self.exps = list(state["m"]), list(state["v"]), list(state["exps"]) if state_bits == 8 else [None] * n
        for w, m, v, e, b in zip(weights, self.m, self.v, self.exps, blocks):
            if any(t.dtype is not kind or t.numel() != w.numel() or not t.is_contiguous() for t in (m, v)):
                raise ValueError("AdamW: moments of another size or type than state_bits says")
            if e is not None and (e.dtype is not torch.uint8 or e.numel() != 2 * b or not e.is_contiguous()):
                raise ValueError("AdamW: two exponents for every %d elements" % B.ADAMW_BLOCK)
        self.plan, self.table = self._table(None, None)

    def _table(self, m_out, v_out):
        at = lambda t: None if t is None else t.data_ptr()   # noqa: E731
        none = [None] * len(self.weights)
        rows = [B.AdamwTensor(at(w), at(g), at(p), at(m), at(v), at(e), at(mo), at(vo), w.numel(), wd, ls) for w, g, p, m, v, e, mo, vo, wd, ls in zip(
            self.weights, self.grads, self.lowp, self.m, self.v, self.exps, m_out or none, v_out or none, self.weight_decay, self.lr_scale)]
        plan, host = B.adamw_table(rows, self.state_bits, B._dtype(self.grads[0]))
        return plan, host.to(self.weights[0].device)

    def step(self, lr, t, beta1=0.9, beta2=0.999, eps=1e-8, seed=0, grad_scale=None):
        """One update; t counts from 1.  seed: the random bits that round 8-bit moments, another one each step.  grad_scale: fp32 device tensor of
        one element that multiplies the gradients, or None."""
        B.codistill_adamw_step(self.plan, self.table, lr, t, beta1, beta2, eps, seed, grad_scale)

    def unpack_plan(self, m_out, v_out):
        """What unpack() needs to write 8-bit moments as values into these lists of bf16 tensors."""
        for outs in (m_out, v_out):
            if len(outs) != len(self.weights) or any(o.dtype is not torch.bfloat16 or o.numel() != w.numel() or not o.is_contiguous()
                                                     for o, w in zip(outs, self.weights)):
                raise ValueError("AdamW: the moments' values are bf16 tensors of the weights' sizes")
        return self._table(m_out, v_out) + ((m_out, v_out),)

    def unpack(self, plan):
        """The values that 8-bit moments stand for, exactly (four significant bits), into the tensors of unpack_plan()."""
        B.codistill_adamw_unpack(plan[0], plan[1])

    def state_dict(self):
        d = {"m": self.m, "v": self.v}
        if self.state_bits == 8:
            d["exps"] = self.exps
        return d
