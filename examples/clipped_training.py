"""A small language model trained with the operators around the step.

    python examples/clipped_training.py

Embedding, one hidden layer, head; next-token prediction on sequences of a
made-up language.  Every parameter lies in one Session; per step:

  * the lookup reads the table's bf16 weights in the Session, scaled by
    sqrt(dim); padded places (id -1) are masked;
  * two micro-batches: the table's gradient is written, then accumulated,
    straight into its part of the Session's flat gradient, the others are
    summed in fp32;
  * one clip takes the norm over all of them (unscaled by the Session's loss
    scale, read on the device), scales the table's gradient in place and rounds
    the fp32 sums into their parts of the flat gradient;
  * the optimizer step follows, skipping by the clip's found_inf, with no
    prepass of its own.

Nothing in the loop waits for the device.  A save window of 4 steps runs in
the middle; the checkpoint restored from it equals the state on the device.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2511_07035_amd import GradList, GradResult, Session, embedding  # noqa: E402

VOCAB, DIM, BATCH, LENGTH = 500, 64, 16, 33
LOSS_SCALE = 256.0


def sequences(gen, follow):
    """[2, BATCH, LENGTH] ids of a language where each token has 4 likely
    followers; the ends of some sequences are padding."""
    ids = torch.empty(2, BATCH, LENGTH, dtype=torch.int64, device="cuda")
    ids[..., 0] = torch.randint(0, VOCAB, (2, BATCH), generator=gen, device="cuda")
    for k in range(1, LENGTH):
        pick = torch.randint(0, 4, (2, BATCH), generator=gen, device="cuda")
        ids[..., k] = follow[ids[..., k - 1], pick]
    ends = torch.randint(LENGTH // 2, LENGTH + 8, (2, BATCH, 1), generator=gen, device="cuda")
    return torch.where(torch.arange(LENGTH, device="cuda") < ends, ids, torch.full_like(ids, -1))


def main(steps=60, window_at=20, K=4, lr=3e-3, max_norm=0.2, verbose=True):
    """Returns the losses, the norms before clipping and the clip coefficients
    of all steps, and whether the restored checkpoint equals the device state."""
    sizes = [VOCAB * DIM, DIM * DIM, VOCAB * DIM]
    n = sum(sizes)
    clipped = GradResult()
    sess = Session(n, ring_bytes=4 << 20, init_scale=LOSS_SCALE, found_inf=clipped.found_inf, grad_norm=False)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    try:
        with torch.cuda.stream(sess.compute):
            follow = torch.randint(0, VOCAB, (VOCAB, 4), generator=gen, device="cuda")
            sess.master.normal_(0.0, 0.08, generator=gen)
            sess.weight.copy_(sess.master)
            table, hidden, head = (w.view(-1, DIM).detach().requires_grad_() for w in torch.split(sess.weight, sizes))
            g_table, g_hidden, g_head = torch.split(sess.grad, sizes)
            sums = [torch.zeros(DIM, DIM, device="cuda"), torch.zeros(VOCAB, DIM, device="cuda")]
            grads = GradList([g_table, *sums], [None, g_hidden, g_head], stream=sess.compute)
            losses, norms, coefs = [], [], []
            for step in range(steps):
                if step == window_at:
                    sess.begin_window([n * k // K // 8 * 8 for k in range(K)] + [n])
                sess.backward_begin()
                batch = sequences(gen, follow)
                loss_sum = torch.zeros((), device="cuda")
                for s in sums:
                    s.zero_()
                for micro in range(2):
                    ids, want = batch[micro, :, :-1], batch[micro, :, 1:]
                    x = embedding(table, ids, scale=DIM ** 0.5, grad_weight=g_table.view(VOCAB, DIM),
                                  accumulate=micro > 0)
                    h = torch.tanh(x.reshape(-1, DIM) @ hidden)
                    loss = torch.nn.functional.cross_entropy((h @ head.t()).float(), want.reshape(-1), ignore_index=-1)
                    (loss * (LOSS_SCALE / 2)).backward()
                    for w, s in zip((hidden, head), sums):
                        s += w.grad
                        w.grad = None
                    loss_sum += loss.detach() / 2
                r = grads.clip(max_norm, scale=sess, result=clipped)
                sess.step(lr)
                losses.append(loss_sum)
                norms.append(r.norm.clone())
                coefs.append(r.coef.clone())
                if step == window_at + K - 1:
                    sess.drain()
                    meta = sess.restore()
                    state = sess.state_to_host()
                    equal = all(np.array_equal(a.view(np.uint32), b.view(np.uint32))
                                for a, b in zip(sess.arena_state(), state[:3]))
                    if verbose:
                        print(f"checkpoint of step {meta.t}: equal to the device state: {equal}", flush=True)
            losses, norms, coefs = (torch.stack(x).flatten().tolist() for x in (losses, norms, coefs))
        if verbose:
            for k in range(0, steps, 10):
                print(f"step {k}: loss {losses[k]:.3f}, norm {norms[k]:.3f}, coefficient {coefs[k]:.3f}")
        return losses, norms, coefs, equal
    finally:
        sess.close()


if __name__ == "__main__":
    main()
