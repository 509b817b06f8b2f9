"""Trains a sequence layer on the GPU and serves it token by token.

Sequences of random ids, each with one of a few marker ids near its start; the
last state has to tell which marker it was, so the recurrence must carry it
over the rest of the sequence.  Per step: token rows looked up and projected,
the gated recurrence over the ragged batch (checkpoints in 8 bits), a linear
head and its loss in PyTorch, then the backward: recurrence from the
checkpoints, the projection's weight gradient from the checkpoint of its
input, the table's rows updated by row-wise Adagrad where they were looked up.
Afterwards the trained layer reads whole sequences once as prompts and once
token by token from a pool of states, which must agree.

    python examples/sequence_training.py [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2112_02752_amd as emb  # noqa: E402

ROWS, DIM, HIDDEN, MARKERS, SEQS, LONGEST = 5000, 64, 96, 8, 64, 60


def make_batch(g):
    """Ragged sequences of 5 to LONGEST ids, some marker among each one's first five."""
    lens = torch.randint(5, LONGEST + 1, (SEQS,), generator=g)
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(lens, 0)])
    ids = torch.randint(MARKERS, ROWS, (int(offsets[-1]),), generator=g)
    labels = torch.randint(0, MARKERS, (SEQS,), generator=g)
    ids[offsets[:-1] + torch.randint(0, 5, (SEQS,), generator=g)] = labels
    return emb.Batch(offsets.int().cuda(), ids.cuda(), SEQS), labels.cuda()


def train(steps=300, say=print):
    g = torch.Generator().manual_seed(1)
    torch.manual_seed(1)
    dev = dict(device="cuda")
    tables = emb.Tables(torch.randn((ROWS, DIM), generator=g).cuda() * 0.1, [0, ROWS])
    master = torch.randn((DIM, 3 * HIDDEN), generator=g).cuda() * DIM ** -0.5    # fp32 weights; the layer's are bf16
    weight = master.bfloat16()
    bias = torch.linspace(1.0, 4.0, HIDDEN, **dev)                               # gates that remember 4 to 50 steps
    head = (torch.randn((HIDDEN, MARKERS), generator=g) * HIDDEN ** -0.5).cuda().requires_grad_()
    most = SEQS * LONGEST
    layer = emb.SequenceLayer(tables, weight, bias, most, SEQS, scale=DIM ** 0.5, opt="adagrad", lr=0.1,
                              state=torch.zeros(ROWS, **dev))
    y, dy = (torch.zeros((most, HIDDEN), dtype=torch.bfloat16, **dev) for _ in range(2))
    h_last = torch.empty((SEQS, HIDDEN), **dev)
    dweight, dbias = torch.empty_like(master), torch.empty_like(bias)
    opt = torch.optim.Adam([master, bias, head], lr=5e-3)
    losses = []
    for step in range(steps):
        batch, labels = make_batch(g)
        n = batch.indices.numel()
        layer.forward(batch, y[:n], h_last)
        top = h_last.detach().requires_grad_()
        loss = torch.nn.functional.cross_entropy(top @ head, labels)
        opt.zero_grad()
        loss.backward()
        layer.backward(batch, dy[:n], dweight, dbias, dh_last=top.grad)
        master.grad, bias.grad = dweight, dbias
        opt.step()
        weight.copy_(master)
        losses.append(loss.detach())
        if step % 50 == 0 or step == steps - 1:
            right = float(((top @ head).argmax(1) == labels).float().mean())
            say(f"step {step:4d}  loss {float(losses[-1]):.4f}  right {right:.2f}")
    layer.tokens.check()
    return layer, head, [float(x) for x in losses], g


def serve(layer, head, g, say=print):
    """The same sequences as prompts and token by token; largest difference of the states."""
    batch, labels = make_batch(g)
    n = batch.indices.numel()
    y = torch.empty((n, HIDDEN), dtype=torch.bfloat16, device="cuda")
    whole = torch.empty((SEQS, HIDDEN), device="cuda")
    layer.forward(batch, y, whole, train=False)
    offsets = batch.offsets.cpu().tolist()
    pool = torch.zeros((2 * SEQS, HIDDEN), device="cuda")
    slots = torch.randperm(2 * SEQS, generator=g)[:SEQS].int().cuda()
    off = 0.0
    for t in range(max(b - a for a, b in zip(offsets, offsets[1:]))):
        rows = [m for m in range(SEQS) if offsets[m] + t < offsets[m + 1]]
        at = torch.tensor([offsets[m] + t for m in rows], device="cuda")
        now = emb.Batch(torch.arange(len(rows) + 1, dtype=torch.int32, device="cuda"), batch.indices[at], len(rows))
        out = torch.empty((len(rows), HIDDEN), dtype=torch.bfloat16, device="cuda")
        layer.step(now, pool, out, slots=slots[rows].contiguous())
        off = max(off, float((out.float() - y[at].float()).abs().max()))
    states = pool[slots.long()]
    right = float(((states @ head).argmax(1) == labels).float().mean())
    say(f"served token by token: right {right:.2f}, states within {float((states - whole).abs().max()):.2e} of the prompt's,"
        f" outputs within {off:.2e}")
    return float((states - whole).abs().max()), right


if __name__ == "__main__":
    trained, linear, _, gen = train(int(sys.argv[1]) if len(sys.argv) > 1 else 300)
    serve(trained, linear.detach(), gen)
