"""A prefetch head from learning to serving.

The early-exit head approximates a model's next-token distribution from an intermediate hidden
state.  Here it is learned from a teacher's top logits (tfe_distill_loss_grad), laid out in 8 bits
(tfe_quantize), and answers a batch: logits of each step's hidden states (tfe_quantized_linear),
one token a row drawn from them (tfe_sample), and the phrases that end at the drawn token injected
into the hidden states (tfe_lookup_inject).

    python examples/head_from_teacher.py [--vocab 2000] [--dim 256] [--steps 60]

The teacher is a random projection; hidden states and phrases are seeded draws."""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_07388_amd import tfe  # noqa: E402

F32, BF16 = tfe.TFE_F32, tfe.TFE_BF16


def stream():
    return torch.cuda.current_stream().cuda_stream


def space(size):
    return torch.empty(max(16, size), dtype=torch.uint8, device="cuda")


def learn(hidden, teacher_ids, teacher_logits, vocab, steps, rate, tau=2.0):
    """W [vocab x dim] by Adam on the mean distillation loss; the losses."""
    rows, dim = hidden.shape
    w = torch.zeros((vocab, dim), device="cuda")
    adam = torch.optim.Adam([w], lr=rate)
    loss, lse = (torch.empty(rows, device="cuda") for _ in range(2))
    weight = torch.full((rows,), 1.0 / rows, device="cuda")
    work = space(tfe.tfe_distill_workspace(rows, vocab))
    means = []
    for _ in range(steps):
        logits = hidden @ w.t()
        # The gradient takes the logits' place.
        tfe.tfe_distill_loss_grad(logits, F32, vocab, rows, vocab, teacher_ids, teacher_logits, F32,
                                  teacher_ids.shape[1], tau, weight, loss, lse, logits, vocab, work,
                                  work.numel(), stream())
        means.append(loss.mean())
        w.grad = logits.t().contiguous() @ hidden
        adam.step()
    return w, torch.stack(means).cpu().numpy()


def layout(w):
    """Codes and scales of a projection, blocks of 128 x 128."""
    rows, dim = w.shape
    blocks = -(-dim // 128)
    codes = torch.empty((rows, blocks * 128), dtype=torch.uint8, device="cuda")
    scales = torch.empty((-(-rows // 128), -(-blocks // 4) * 4), dtype=torch.uint8, device="cuda")
    tfe.tfe_quantize(w, F32, dim, rows, dim, 128, codes, scales, stream())
    return codes, scales


def phrase_table(tokens, values):
    """Every 2-gram of the given rows of tokens, with a value row each."""
    grams = np.unique(np.concatenate([tokens[:, i:i + 2] for i in range(tokens.shape[1] - 1)]), axis=0)
    grams = np.ascontiguousarray(grams[:values.shape[0]], np.int32)
    lens = np.full(len(grams), 2, np.uint8)
    desc = tfe.make_desc(grams, lens, 2, 2, 1 << 18, values, values.shape[1], F32, True)
    return tfe.tfe_table_load(desc, stream()), len(grams)


def answer(hidden, codes, scales, table, vocab, steps, seed):
    """`steps` steps of a batch: (tokens [rows x steps + 1], probabilities, matched positions)."""
    rows, dim = hidden.shape
    rng = torch.Generator(device="cuda").manual_seed(seed)
    logits = torch.empty((rows, vocab), device="cuda")
    linear = space(tfe.tfe_quantized_workspace(rows, dim))
    draw = space(tfe.tfe_sample_workspace(rows, vocab))
    temperature = torch.full((rows,), 0.8, device="cuda")
    top_k = torch.full((rows,), 50, dtype=torch.int32, device="cuda")
    top_p = torch.full((rows,), 0.95, device="cuda")
    window = torch.zeros((rows, 2), dtype=torch.int32, device="cuda")
    token, slot = (torch.empty(rows, dtype=torch.int32, device="cuda") for _ in range(2))
    prob = torch.empty(rows, device="cuda")
    hit = torch.empty(rows, dtype=torch.uint8, device="cuda")
    tokens, probs, hits = [window[:, 1].clone()], [], 0
    for _ in range(steps):
        tfe.tfe_quantized_linear(hidden, F32, dim, codes, scales, rows, vocab, dim, logits, F32, vocab,
                                 linear, linear.numel(), stream())
        u = torch.rand(rows, generator=rng, device="cuda")
        tfe.tfe_sample(logits, F32, vocab, rows, vocab, temperature, top_k, top_p, None, u, token, prob,
                       draw, draw.numel(), stream())
        window = torch.stack([window[:, 1], token], 1).contiguous()
        # The phrase that ends at the drawn token goes into the next hidden states.
        hidden = hidden.roll(1, 0).contiguous()
        tfe.tfe_lookup_inject(table, window, rows, 1, 1, hidden, hidden, hit, slot, None,
                              tfe.TFE_GATE_SIGMOID, 1.0, stream())
        tokens.append(token.clone())
        probs.append(prob.clone())
        hits += int(hit.sum())
    return torch.stack(tokens, 1).cpu().numpy(), torch.stack(probs, 1).cpu().numpy(), hits


def main(vocab=2000, dim=256, rows=512, steps=60, batch=16, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    hidden = torch.randn((rows, dim), generator=g, device="cuda")
    target = torch.randn((vocab, dim), generator=g, device="cuda") * (6.0 / dim ** 0.5)
    top = (hidden @ target.t()).topk(32, dim=1)
    w, losses = learn(hidden, top.indices.int().contiguous(), top.values.contiguous(), vocab, steps, rate=0.03)
    codes, scales = layout(w)
    exact = hidden[:batch] @ w.t()
    # Phrases from a first answer, so that the second one meets some.
    table, _ = phrase_table(np.zeros((1, 2), np.int32), torch.zeros((1, dim), device="cuda"))
    first, _, _ = answer(hidden[:batch], codes, scales, table, vocab, 12, seed)
    tfe.tfe_table_free(table)
    values = torch.randn((512, dim), generator=g, device="cuda") * 0.02
    table, phrases = phrase_table(first, values)
    tokens, probs, hits = answer(hidden[:batch], codes, scales, table, vocab, 12, seed)
    torch.cuda.synchronize()
    tfe.tfe_table_free(table)
    return {"losses": losses, "tokens": tokens, "probs": probs, "hits": hits, "phrases": phrases,
            "best": exact.argmax(1).cpu().numpy(), "teacher": top.indices[:batch, 0].cpu().numpy()}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("vocab", 2000), ("dim", 256), ("rows", 512), ("steps", 60), ("batch", 16), ("seed", 1)):
        ap.add_argument("--" + name, type=int, default=default)
    r = main(**vars(ap.parse_args()))
    print("mean loss %.3f -> %.3f over %d steps" % (r["losses"][0], r["losses"][-1], len(r["losses"])))
    print("teacher's first choice learned for %d of %d rows" % ((r["best"] == r["teacher"]).sum(), len(r["best"])))
    print("drawn: %s ..., mean probability %.2f" % (r["tokens"][0, 1:7].tolist(), r["probs"].mean()))
    print("%d phrases, %d positions matched" % (r["phrases"], r["hits"]))
