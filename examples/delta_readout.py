"""A readout whose memory is a matrix per head: features of a spiking stack -> queries, keys, values and gates -> gated delta rule -> logits.

    x [T, B, F] --8 bits--> product --> query, key, value, gate, write
    query, key --norm of each head, rotation by time--> gated delta rule with value, gate, write --> norm, 8 bits --> product --> logits

Whole sequences are taken a chunk of steps at a time, forwards and backwards; serving keeps a pool of states and answers after every frame.  Gains of Dk^-1/2 make keys of
length 1, which the delta rule wants.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_13810_amd import api  # noqa: E402

EPS = 1e-5


class DeltaReadout:
    def __init__(self, features, k_heads, v_heads, dk, dv, classes, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda n, k: torch.randn(n, k, generator=g, device=device) / k ** 0.5
        self.F, self.hk, self.hv, self.dk, self.dv, self.classes, self.dtype = features, k_heads, v_heads, dk, dv, classes, dtype
        self.widths = [k_heads * dk, k_heads * dk, v_heads * dv, v_heads, v_heads]
        self.N, self.D = sum(self.widths), v_heads * dv
        self.w_in, self.w_out = rand(self.N, features), rand(classes, self.D)
        self.b_in = torch.zeros(self.N, device=device)
        self.b_in[-2 * v_heads:-v_heads] = 3.0                    # memories fade slowly at first
        self.gain_q = torch.full((dk,), dk ** -0.5, device=device)
        self.gain_k = self.gain_q.clone()
        self.gain = torch.ones(self.D, device=device)

    def lay_out(self):
        """The weights in 8 bits, the same values along their rows and along their columns.  Once per update."""
        self.in8 = api.tac_quantize(self.w_in, tiles=True, columns=True)
        self.out8 = api.tac_quantize(self.w_out, tiles=True, columns=True)

    def parts(self, rows):
        """Slices of a product's rows [.., N]: query, key [.., k_heads, Dk], value [.., v_heads, Dv], gate, write [.., v_heads]."""
        q, k, v, gate, write = rows.split(self.widths, -1)
        return q.unflatten(-1, (self.hk, self.dk)), k.unflatten(-1, (self.hk, self.dk)), v.unflatten(-1, (self.hv, self.dv)), gate, write

    def heads(self, rows, positions):
        q, k = self.parts(rows)[:2]
        return api.tac_head_norm(q, k, self.gain_q, self.gain_k, eps=EPS, positions=positions)

    def forward(self, x, lengths=None, h0=None):
        """x [T, B, F].  Returns logits [T, B, classes], the last states, and what backward() reads."""
        T, B = x.shape[:2]
        positions = torch.arange(T, dtype=torch.int32, device=x.device).repeat_interleave(B)
        x8 = api.tac_quantize(x.reshape(T * B, self.F).to(self.dtype))["rows"]
        rows = api.tac_scaled_product(*x8, *self.in8["rows"], self.F, bias=self.b_in, dtype=self.dtype)
        qk = {n: t.view(T, B, self.hk, self.dk) for n, t in self.heads(rows, positions).items()}
        value, gate, write = self.parts(rows.view(T, B, self.N))[2:]
        scan = api.tac_delta_scan(qk["q"], qk["k"], value, gate, write, lengths=lengths, h0=h0, want_kept=True)
        norm = api.tac_residual_norm(scan["out"].view(T * B, self.D), None, self.gain, eps=EPS, want_y=False, want_scaled=True, want_rstd=True)
        logits = api.tac_scaled_product(*norm["scaled"], *self.out8["rows"], self.D, dtype=torch.float32).view(T, B, self.classes)
        return logits, scan["h_last"], (x8, rows, positions, qk, lengths, scan, norm)

    def backward(self, kept, grad_logits, want_bias=True):
        """Gradients of the weights, of x [T * B, F] and of h0 from that of the logits [T, B, classes].  The bias's is torch's sum, which does not belong into a captured graph."""
        x8, rows, positions, qk, lengths, scan, norm = kept
        T, B = scan["out"].shape[:2]
        R = T * B
        gl = api.tac_quantize(grad_logits.reshape(R, self.classes), columns=True)
        y_cols = api.tac_quantize(norm["scaled"], cols=self.D, rows=False, columns=True)["columns"]
        grad_w_out = api.tac_scaled_product(*gl["columns"], *y_cols, R, dtype=torch.float32)
        grad_y = api.tac_scaled_product(*gl["rows"], *self.out8["columns"], self.classes, dtype=self.dtype)
        back = api.tac_residual_norm_backward(scan["out"].view(R, self.D), self.gain, norm["rstd"], grad_y)
        grad_rows = torch.empty_like(rows)                        # every part's gradient into its own slice
        value, gate, write = self.parts(rows.view(T, B, self.N))[2:]
        gq, gk, gv, gg, gw = self.parts(grad_rows.view(T, B, self.N))
        d = api.tac_delta_scan_backward(qk["q"], qk["k"], value, gate, write, scan["states"], scan["updates"], back["grad_x"].view_as(scan["out"]),
                                        lengths=lengths, grad_value=gv, grad_gate=gg, grad_write=gw)
        q, k = self.parts(rows)[:2]
        h = api.tac_head_norm_backward(q, k, self.gain_q, self.gain_k, d["grad_query"].view(R, self.hk, self.dk), d["grad_key"].view(R, self.hk, self.dk),
                                       eps=EPS, positions=positions, grad_query=gq.view(R, self.hk, self.dk), grad_key=gk.view(R, self.hk, self.dk))
        gb = api.tac_quantize(grad_rows, columns=True)
        x_cols = api.tac_quantize(x8, cols=self.F, rows=False, columns=True)["columns"]
        bias = dict(b_in=grad_rows.float().sum(0)) if want_bias else {}
        return dict(bias, w_out=grad_w_out, gain=back["grad_gain"], gain_q=h["grad_gain_q"], gain_k=h["grad_gain_k"],
                    w_in=api.tac_scaled_product(*gb["columns"], *x_cols, R, dtype=torch.float32),
                    x=api.tac_scaled_product(*gb["rows"], *self.in8["columns"], self.N, dtype=torch.float32), h0=d["grad_h0"])

    def step(self, x, positions, pool, slots):
        """One frame of B running sequences: x [B, F], their times [B], their states at `slots` of `pool`.  Returns logits [B, classes]."""
        x8 = api.tac_quantize(x.to(self.dtype))["rows"]
        rows = api.tac_scaled_product(*x8, *self.in8["rows"], self.F, bias=self.b_in, dtype=self.dtype)
        qk = self.heads(rows, positions)
        out = api.tac_delta_step(qk["q"], qk["k"], *self.parts(rows)[2:], pool, slots)
        y8 = api.tac_residual_norm(out.view(-1, self.D), None, self.gain, eps=EPS, want_y=False, want_scaled=True)["scaled"]
        return api.tac_scaled_product(*y8, *self.out8["rows"], self.D, dtype=torch.float32)


def main(steps=150, T=20, B=64, pairs=4, symbols=8, device="cuda:0"):
    """Recall: a sequence shows pairs (symbol, answer) in frames of spikes and then asks for one symbol's answer, which the memory has to hold."""
    g = torch.Generator(device=device).manual_seed(7)
    F = 2 * 16 * symbols
    net = DeltaReadout(F, 2, 4, 32, 32, symbols, device=device)
    net.lay_out()

    def batch():
        key = torch.stack([torch.randperm(symbols, generator=g, device=device)[:pairs] for _ in range(B)])
        answer = torch.randint(symbols, (B, pairs), generator=g, device=device)
        asked = torch.randint(pairs, (B,), generator=g, device=device)
        x = torch.zeros(pairs + 1, B, 2, symbols, 16, device=device)
        at = torch.arange(B, device=device)
        for i in range(pairs):
            x[i, at, 0, key[:, i]] = 1.0
            x[i, at, 1, answer[:, i]] = 1.0
        x[pairs, at, 0, key[at, asked]] = 1.0
        return (x.flatten(2) * (torch.rand(pairs + 1, B, F, generator=g, device=device) < 0.9)), answer[at, asked]

    losses = []
    for i in range(steps):
        x, labels = batch()
        logits, _, kept = net.forward(x)
        p = torch.softmax(logits[-1], 1)
        grad = torch.zeros_like(logits)
        grad[-1] = (p - torch.nn.functional.one_hot(labels, symbols)) / B
        grads = net.backward(kept, grad)
        for name in ("w_in", "w_out", "b_in", "gain", "gain_q", "gain_k"):
            rate = 0.05 if name.startswith("gain_") else 0.5
            w = getattr(net, name)
            w -= rate * grads[name]
        net.lay_out()
        losses.append(float(-torch.log(p.gather(1, labels[:, None])).mean()))
        if i % 25 == 0:
            print("step %d: loss %.3f" % (i, losses[-1]), flush=True)
    return losses


if __name__ == "__main__":
    main()
