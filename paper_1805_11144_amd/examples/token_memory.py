"""A token front end, trained, served and read out by spiking neurons.

    python -m paper_1805_11144_amd.examples.token_memory

Sequences mix a few symbols to be remembered with many distractors; at every step the answer is the symbol
seen last.  Token vectors from a table (`embed`) give, by one matrix each, the value and the gate of a gated
lowpass, which learns to open at a symbol and to hold through distractors; a third matrix reads its state.
Training takes the gradient back through the filter (`gated_lowpass_grad`) to the matrices, which learn by
orthogonalised updates, and to the table (`embed_grad`).  Serving answers one token at a time
(`gated_lowpass_step`) from a cache of states.  At last the answers are the feed of an ensemble of spiking
neurons, whose decoded output is read through a synapse.
"""
from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import torch

import paper_1805_11144_amd as M


class TokenMemory:
    """Table [vocab, dim], matrices [dim, dim] of the filter's values and gates, readout [symbols, dim]."""

    def __init__(self, vocab=512, symbols=8, dim=128, seed=0, device="cuda"):
        gen = torch.Generator().manual_seed(seed)
        self.scale, self.gate_bias = dim ** 0.5, 1.0
        self.table = (torch.randn(vocab, dim, generator=gen) / self.scale).to(device)
        self.values, self.gates = (torch.randn(2, dim, dim, generator=gen) / dim ** 0.5).to(device)
        self.readout = (torch.randn(symbols, dim, generator=gen) / dim ** 0.5).to(device)
        self.momenta = [torch.zeros_like(w) for w in (self.values, self.gates, self.readout)]

    def _inputs(self, tokens):
        x = M.embed(tokens, self.table, scale=self.scale)
        return x, torch.matmul(x, self.values.T), torch.matmul(x, self.gates.T) + self.gate_bias

    def answers(self, tokens):
        """Logits [batch, steps, symbols] of whole sequences."""
        _, v, g = self._inputs(tokens)
        return torch.matmul(M.gated_lowpass(v, g)[0], self.readout.T)

    def train_step(self, tokens, targets, rate=0.02, table_rate=2.0):
        """One update from tokens and targets [batch, steps] (both int); returns the mean cross entropy."""
        x, v, g = self._inputs(tokens)
        y, _, kept = M.gated_lowpass(v, g, keep=True)
        logits = torch.matmul(y, self.readout.T)
        log_p = logits - torch.logsumexp(logits, -1, keepdim=True)
        loss = -log_p.gather(-1, targets[..., None]).mean()
        d = torch.exp(log_p)
        d.scatter_add_(-1, targets[..., None], torch.full_like(log_p[..., :1], -1.0))
        d /= targets.numel()

        def flat(t):
            return t.reshape(-1, t.shape[-1])
        dv, dg, _ = M.gated_lowpass_grad(v, g, kept, torch.matmul(d, self.readout))
        grads = [flat(dv).T @ flat(x), flat(dg).T @ flat(x), flat(d).T @ flat(y)]
        dx = torch.matmul(dv, self.values) + torch.matmul(dg, self.gates)
        M.embed_grad(tokens, dx, scale=-table_rate * self.scale, out=self.table, accumulate=True)
        for w, m, grad in zip((self.values, self.gates, self.readout), self.momenta, grads):
            M.orthogonal_update(w, m, grad, rate=rate, momentum_decay=0.9)
        return loss

    def serve(self, tokens, state, slots):
        """Logits [rows, symbols] of one more token of each sequence, whose states are state[slots]."""
        _, v, g = self._inputs(tokens)
        return M.gated_lowpass_step(v, g, state, slots=slots) @ self.readout.T


def sequences(batch, steps, vocab, symbols, gen, device="cuda"):
    """(tokens, targets): tokens below `symbols` are to be remembered, one in eight; the first one is one."""
    tokens = torch.randint(symbols, vocab, (batch, steps), generator=gen)
    seen = torch.rand(batch, steps, generator=gen) < 0.125
    seen[:, 0] = True
    tokens[seen] = torch.randint(symbols, (int(seen.sum()),), generator=gen)
    last = torch.where(seen, torch.arange(steps), 0).cummax(1).values
    return tokens.to(device), tokens.gather(1, last).to(device)


def spiking_readout(p, neurons=400, synapse=0.01, hold=20, seed=0):
    """Answers p [batch, n, symbols] shown for `hold` steps of 1 ms each to an ensemble of LIF neurons; its
    decoded output, filtered, at the end of each."""
    batch, n, symbols = p.shape
    rng = np.random.default_rng(seed)

    def directions(k):
        x = rng.standard_normal((k, symbols))
        return x / np.linalg.norm(x, axis=1, keepdims=True)
    points = directions(1000) * rng.uniform(0, 1, (1000, 1)) ** (1 / symbols)
    model = M.Model()
    node = model.add_node(symbols)
    model.add_ensemble(SimpleNamespace(
        n_neurons=neurons, dims=symbols, neuron_type="lif", tau_rc=0.02, tau_ref=0.002, amplitude=1.0,
        encoders=directions(neurons), max_rates=rng.uniform(200, 400, neurons), intercepts=rng.uniform(-0.9, 0.9, neurons),
        gains=None, biases=None, eval_points=points))
    model.add_connection(SimpleNamespace(pre=("node", node), post=("ens", 0), pre_slice=None, post_slice=None,
                                         function="identity", decoders=None, transform=1.0, synapse=None))
    model.add_probe(SimpleNamespace(target=("ens", 0), synapse=synapse))
    torch.cuda.synchronize()   # the feed is complete before the simulator's stream reads it
    with M.Simulator(model, minibatch=batch, device=p.device.index, probe_capacity_steps=n * hold) as sim:
        sim.run_steps(n * hold, {node: p.repeat_interleave(hold, dim=1).contiguous()})
        return sim.data(0)[:, hold - 1::hold]


def run(updates=150, batch=64, steps=100, vocab=512, symbols=8, seed=0, say=print):
    gen = torch.Generator().manual_seed(seed)
    net = TokenMemory(vocab, symbols, seed=seed)
    losses = [net.train_step(*sequences(batch, steps, vocab, symbols, gen)) for _ in range(updates)]
    losses = torch.stack(losses).cpu().numpy()
    say(f"training: cross entropy {losses[0]:.3f} -> {losses[-1]:.3f} in {updates} updates")
    tokens, targets = sequences(batch, steps, vocab, symbols, gen)
    whole = net.answers(tokens)
    right = float((whole.argmax(-1) == targets).float().mean())
    # one token at a time, the sequences' states in the slots of a larger cache
    slots = torch.randperm(2 * batch, generator=gen)[:batch].to(torch.int32).to(tokens.device)
    state = torch.zeros(2 * batch, net.values.shape[0], device=tokens.device)
    served = torch.stack([net.serve(tokens[:, t], state, slots) for t in range(steps)], 1)
    apart = float((served - whole).abs().max() / whole.abs().max())
    say(f"answers: {right:.3f} right; served one token at a time, within {apart:.1e} of the whole run's")
    shown = torch.softmax(whole[:8, ::5], -1)
    decoded = spiking_readout(shown)
    spiking = float((decoded.argmax(-1) == shown.argmax(-1).cpu().numpy()).mean())
    say(f"spiking readout of {shown.shape[0]} x {shown.shape[1]} answers: {spiking:.3f} agree")
    return SimpleNamespace(losses=losses, right=right, apart=apart, spiking=spiking)


if __name__ == "__main__":
    run()
