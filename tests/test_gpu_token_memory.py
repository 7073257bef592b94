"""GPU: the token front end's example: it learns its task, answers one token at a time as it does on whole
sequences, and spiking neurons show its answers.

Chance is a cross entropy of ln 8 = 2.08 and one answer in eight.  Serving and the whole run compute the same
filter; their products differ in the order of 32-bit sums of 128 terms (1e-5), which passes through the gates."""
import pytest
import torch

from paper_1805_11144_amd.examples import token_memory

pytestmark = pytest.mark.gpu


def test_example_learns_serves_and_spikes():
    r = token_memory.run(say=lambda s: print(s))
    assert r.losses[0] > 1.5 and r.losses[-10:].mean() < 0.5
    assert r.right > 0.85 and r.apart < 1e-3 and r.spiking > 0.9


def test_gradients_of_the_whole_path_against_differences():
    """One update with plain descent on the table: its change is the gradient of the loss in 64 bits."""
    gen = torch.Generator().manual_seed(3)
    net = token_memory.TokenMemory(vocab=40, symbols=4, dim=16, seed=3)
    tokens, targets = token_memory.sequences(5, 30, 40, 4, gen)
    table, values, gates, readout = (t.double().cpu() for t in (net.table, net.values, net.gates, net.readout))
    ids, want = tokens.cpu(), targets.cpu()

    def loss(table):
        x = table[ids] * net.scale
        v, a = x @ values.T, torch.sigmoid(x @ gates.T + net.gate_bias)
        h, out = torch.zeros(5, 16, dtype=torch.float64), []
        for t in range(30):
            h = a[:, t] * h + (1 - a[:, t]) * v[:, t]
            out.append(h)
        logits = torch.stack(out, 1) @ readout.T
        return -(logits.log_softmax(-1).gather(-1, want[..., None])).mean()

    net.train_step(tokens, targets, rate=0.0, table_rate=1.0)
    change = (net.table.double().cpu() - table)
    z = torch.randn(table.shape, generator=gen, dtype=torch.float64)
    slope = float(loss(table + 1e-5 * z) - loss(table - 1e-5 * z)) / 2e-5
    assert abs(slope + float((change * z).sum())) <= 1e-4 * float((change * z).abs().sum())
