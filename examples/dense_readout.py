"""A spiking layer with a dense recurrent readout: trained on whole sequences, then run frame by frame.

    spikes [T, B, F] --8 bits--> product --> gate, value [T, B, D] --> gated recurrence --> + value, norm, 8 bits --> product --> logits

The readout's matrices are products of 8-bit matrices with a power of two per 128 values; what the backward pass needs of the forward pass is
kept in 8 bits (the spikes and the normed features), as the sum behind the recurrence, and as every 16th state.  Gradients go on into the
spiking layer (tac_stack_backward).  Serving keeps the membrane and a pool of states and answers after every frame.

    python examples/dense_readout.py            # synthetic classes: a rate per pixel each
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2603_13810_amd import api  # noqa: E402

EPS = 1e-5


class DenseReadout:
    def __init__(self, features, width, classes, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        rand = lambda n, k: torch.randn(n, k, generator=g, device=device) / k ** 0.5
        self.F, self.D, self.classes, self.dtype = features, width, classes, dtype
        self.w_in, self.w_out = rand(2 * width, features), rand(classes, width)
        self.b_in = torch.zeros(2 * width, device=device)
        self.b_in[:width] = 1.0                                   # leaks start between a half and one
        self.gain = torch.ones(width, device=device)

    def lay_out(self):
        """The weights in 8 bits, in tiles: the same values along their rows and along their columns.  Once per update."""
        self.in8 = api.tac_quantize(self.w_in, tiles=True, columns=True)
        self.out8 = api.tac_quantize(self.w_out, tiles=True, columns=True)

    def forward(self, spikes, h0=None):
        """spikes [T, B, F] (0 / 1).  Returns logits [T, B, classes], the last states, and what backward() reads."""
        T, B, D = spikes.shape[0], spikes.shape[1], self.D
        x8 = api.tac_quantize(spikes.reshape(T * B, self.F).to(self.dtype))["rows"]
        both = api.tac_scaled_product(*x8, *self.in8["rows"], self.F, bias=self.b_in, dtype=self.dtype).view(T, B, 2 * D)
        gate, value = both[..., :D], both[..., D:]
        scan = api.tac_gated_scan(gate, value, h0=h0, want_states=True)
        norm = api.tac_residual_norm(scan["out"].view(T * B, D), value.reshape(T * B, D), self.gain, eps=EPS, want_y=False,
                                     want_scaled=True, want_rstd=True)
        logits = api.tac_scaled_product(*norm["scaled"], *self.out8["rows"], D, dtype=torch.float32).view(T, B, self.classes)
        return logits, scan["h_last"], (x8, both, scan["states"], norm)

    def backward(self, kept, grad_logits):
        """Gradients of the weights, and of the spikes [T * B, F], from that of the logits [T, B, classes]."""
        x8, both, states, norm = kept
        (T, B), D = both.shape[:2], self.D
        R = T * B
        gate, value = both[..., :D], both[..., D:]
        gl = api.tac_quantize(grad_logits.reshape(R, self.classes), columns=True)
        y_cols = api.tac_quantize(norm["scaled"], cols=D, rows=False, columns=True)["columns"]
        grad_out = api.tac_scaled_product(*gl["columns"], *y_cols, R, dtype=torch.float32)
        grad_y = api.tac_scaled_product(*gl["rows"], *self.out8["columns"], self.classes, dtype=self.dtype)
        back = api.tac_residual_norm_backward(norm["h"], self.gain, norm["rstd"], grad_y)
        grad_both = torch.empty_like(both)
        api.tac_gated_scan_backward(gate, value, states, back["grad_x"].view(T, B, D), grad_gate=grad_both[..., :D],
                                    grad_value=grad_both[..., D:], want_grad_h0=False)
        grad_both[..., D:] += back["grad_x"].view(T, B, D)       # the value's other way, past the recurrence
        gb = api.tac_quantize(grad_both.view(R, 2 * D), columns=True)
        x_cols = api.tac_quantize(x8, cols=self.F, rows=False, columns=True)["columns"]
        return dict(w_out=grad_out, gain=back["grad_gain"], b_in=grad_both.float().sum((0, 1)),
                    w_in=api.tac_scaled_product(*gb["columns"], *x_cols, R, dtype=torch.float32),
                    spikes=api.tac_scaled_product(*gb["rows"], *self.in8["columns"], 2 * D, dtype=torch.float32))

    def step(self, spikes, pool, slots):
        """One frame of B running sequences: spikes [B, F], their states at `slots` of `pool`.  Returns logits [B, classes]."""
        D = self.D
        x8 = api.tac_quantize(spikes.to(self.dtype))["rows"]
        both = api.tac_scaled_product(*x8, *self.in8["rows"], self.F, bias=self.b_in, dtype=self.dtype)
        out = api.tac_gated_step(both[:, :D], both[:, D:], pool, slots)
        y8 = api.tac_residual_norm(out, both[:, D:], self.gain, eps=EPS, want_h=False, want_y=False, want_scaled=True)["scaled"]
        return api.tac_scaled_product(*y8, *self.out8["rows"], D, dtype=torch.float32)


class Network:
    """One spiking layer (stride 2, a membrane update per frame) in front of the readout."""

    def __init__(self, side, channels, width, classes, beta=0.9, device="cuda:0", dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device=device).manual_seed(seed + 1)
        self.side, self.channels, self.beta, self.device = side, channels, beta, device
        self.w_conv = torch.randn(channels, 1, 3, 3, generator=g, device=device) * (2 / 9) ** 0.5
        self.out_side = (side + 1) // 2
        self.readout = DenseReadout(channels * self.out_side ** 2, width, classes, dtype, device, seed)
        self.update({})

    def desc(self, T, B):
        return api.make_desc(T, B, 1, self.side, self.side, self.channels, K=1, beta=self.beta, theta=1.0, mode=api.TAC_PER_STEP, stride=2)

    def update(self, grads, rate=0.0):
        for name, g in grads.items():
            w = self.w_conv if name == "w_conv" else getattr(self.readout, name)
            w -= rate * g
        self.w_prepared = api.tac_prepare_weights(self.desc(1, 1), self.w_conv)
        self.readout.lay_out()

    def spikes_of(self, frames, v=None, trace=False):
        """frames uint8 [T, B, 1, side, side] -> spikes [T, B, F] and what the stack's backward pass reads."""
        T, B = frames.shape[:2]
        layer = dict(desc=self.desc(T, B), w_prepared=self.w_prepared, v_inout=v)
        if trace:
            layer["v_trace"] = torch.empty((T, B, self.channels, self.out_side, self.out_side), device=self.device)
        stack, outs = api.make_stack([layer])
        packed = api.tac_pack_spikes(frames)
        api.tac_stack_forward(stack, packed)
        return api.tac_unpack_spikes(outs[0], self.out_side).view(T, B, self.readout.F), (stack, packed, layer)

    def train_step(self, frames, labels, rate):
        """One step of plain gradient descent on the cross entropy of the logits' mean over time.  Returns the loss."""
        spikes, (stack, packed, layer) = self.spikes_of(frames, trace=True)
        logits, _, kept = self.readout.forward(spikes)
        T, B, n = logits.shape
        p = torch.softmax(logits.mean(0), 1)
        wanted = torch.nn.functional.one_hot(labels, n)
        grads = self.readout.backward(kept, ((p - wanted) / (B * T)).expand(T, B, n).contiguous())
        grad_spikes = grads.pop("spikes").view(T, B, self.channels, self.out_side, self.out_side)
        grads["w_conv"] = api.tac_stack_backward(stack, [self.w_conv], packed, grad_spikes, alpha=5.0)[0]["grad_w"]
        self.update(grads, rate)
        return float(-torch.log(p.gather(1, labels[:, None])).mean())


def frames_of(rates, labels, T, generator):
    """0 / 1 frames [T, B, 1, side, side] at the pixel rates [classes, side, side] of each sequence's class."""
    p = rates[labels][None, :, None].expand(T, -1, 1, -1, -1)
    return (torch.rand(p.shape, generator=generator, device=p.device) < p).to(torch.uint8)


def main(steps=60, T=12, B=64, side=16, channels=8, width=128, classes=5, device="cuda:0"):
    g = torch.Generator(device=device).manual_seed(7)
    rates = 0.6 * torch.rand(classes, side, side, generator=g, device=device)
    net = Network(side, channels, width, classes, device=device)
    losses = []
    for i in range(steps):
        labels = torch.randint(classes, (B,), generator=g, device=device)
        losses.append(net.train_step(frames_of(rates, labels, T, g), labels, rate=0.3))
        if i % 10 == 0:
            print("step %d: loss %.3f" % (i, losses[-1]), flush=True)

    # frame by frame: the membrane and the states are carried, rows of a pool in any order
    labels = torch.randint(classes, (B,), generator=g, device=device)
    frames = frames_of(rates, labels, T, g)
    whole = net.readout.forward(net.spikes_of(frames)[0])[0]
    v = torch.zeros(B, channels, net.out_side, net.out_side, device=device)
    pool, slots = torch.zeros(B + 8, width, device=device), torch.randperm(B + 8, generator=g, device=device)[:B].to(torch.int32)
    running = torch.stack([net.readout.step(net.spikes_of(frames[t:t + 1], v)[0][0], pool, slots) for t in range(T)])
    right = float((running.mean(0).argmax(1) == labels).float().mean())
    apart = float((running - whole).abs().max() / whole.abs().max())
    print("frame by frame: %.0f%% right, logits %.1e apart from the whole sequences'" % (100 * right, apart))
    return losses, right, apart


if __name__ == "__main__":
    main()
