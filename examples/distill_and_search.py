"""A student learns next tokens from a teacher's top logits, and answers by beam search.

The teacher is a table of next-token logits of which only the K largest of each row are kept (comet_rows_topk): a sparse
matrix tokens x vocabulary in the library's level storage.  The student, a table of lower rank, is trained on these rows with
comet_distill_forward / comet_distill_backward under automatic differentiation, or with comet_distill_step where there is no
graph to build.  Then it continues prompts with several beams: comet_beam_select picks the continuations and
comet_beam_reorder lets the beams' histories and caches follow.

    python examples/distill_and_search.py [--vocabulary 4001] [--steps 300]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2102_05187_amd as comet  # noqa: E402

TEMPERATURE = 2.0


class Distill(torch.autograd.Function):
    """Losses of the rows of Z against teacher rows (crd, tvals, tlse), differentiable by Z."""

    @staticmethod
    def forward(ctx, Z, crd, tvals, tlse, scale):
        loss, stat = comet.comet_distill_forward(Z, crd, tvals, tlse=tlse, scale=scale)
        ctx.save_for_backward(Z, crd, tvals, tlse, stat)
        ctx.scale = scale
        return loss

    @staticmethod
    def backward(ctx, dloss):
        Z, crd, tvals, tlse, stat = ctx.saved_tensors
        dZ = comet.comet_distill_backward(Z, crd, tvals, stat, tlse=tlse, scale=ctx.scale, dloss=dloss.float().contiguous())
        return dZ, None, None, None, None


def teacher_rows(vocabulary, kept, generator):
    """The teacher's kept logits for every token, with the log-sum-exp of its whole rows."""
    rank = 48
    a, b = (torch.randn((vocabulary, rank), device="cuda", generator=generator) for _ in range(2))
    logits = (a @ b.t()).mul_(6.0 / rank ** 0.5).bfloat16()
    return comet.comet_rows_topk(logits, kept, scale=1.0 / TEMPERATURE, by_coordinate=True)


def as_matrix(crd, values, columns):
    """Kept entries in the order of their coordinates, as a [D, CU] matrix of the library."""
    rows, kept = crd.shape
    pos = torch.arange(rows + 1, dtype=torch.int32, device="cuda") * kept
    size = torch.tensor([rows], dtype=torch.int32, device="cuda")
    return comet.comet_tensor_create([rows, columns], [comet.COMET_D, comet.COMET_CU], [size, pos], [None, crd.reshape(-1)], values.double().reshape(-1))


def train(vocabulary, kept, rank, steps, generator):
    """(input table, output table, losses of the first and the last steps)."""
    crd, tvals, tlse = teacher_rows(vocabulary, kept, generator)
    out = torch.randn((vocabulary, rank), device="cuda", generator=generator).mul_(0.3)
    # a token's first vector is the mean of what it is followed by: the teacher's probabilities times the output table
    p = torch.exp(tvals / TEMPERATURE - tlse[:, None])
    table = comet.comet_spmm(as_matrix(crd, p, vocabulary), out.double()).float()
    table.requires_grad_(), out.requires_grad_()
    optimizer = torch.optim.Adam([table, out], lr=0.03)
    losses = []
    for _ in range(steps):
        x = torch.randint(vocabulary, (512,), device="cuda", generator=generator)
        logits = (table[x] @ out.t()).bfloat16()
        loss = Distill.apply(logits, crd[x], tvals[x], tlse[x], 1.0 / TEMPERATURE).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    with torch.no_grad():
        # the same numbers in one call, for steps without automatic differentiation; the gradient takes the logits' place
        x = torch.arange(min(512, vocabulary), device="cuda")
        logits = (table[x] @ out.t()).bfloat16()
        separate = Distill.apply(logits, crd[x], tvals[x], tlse[x], 1.0 / TEMPERATURE)
        together, _ = comet.comet_distill_step(logits, crd[x], tvals[x], tlse=tlse[x], scale=1.0 / TEMPERATURE, dZ=logits)
        assert torch.allclose(separate, together, rtol=1e-4, atol=1e-5)
    return table.detach(), out.detach(), torch.stack(losses[:10]).mean().item(), torch.stack(losses[-10:]).mean().item()


def search(table, out, prompts, beams, length, end):
    """(scores, tokens) of the beams after `length` steps, best first."""
    batch, rank = prompts.numel(), table.shape[1]
    score = torch.full((batch, beams), -float("inf"), device="cuda")
    score[:, 0] = 0                                                 # one beam to begin with
    last = prompts[:, None].expand(batch, beams).contiguous()
    history = torch.full((batch, beams, length), end, dtype=torch.int32, device="cuda")
    cache = torch.zeros((batch, beams, length, rank), dtype=torch.bfloat16, device="cuda")
    finished = torch.zeros((batch, beams), dtype=torch.bool, device="cuda")
    for step in range(length):
        hidden = table[last]
        cache[:, :, step] = hidden.bfloat16()
        logits = (hidden @ out.t()).bfloat16()
        score, parent, token = comet.comet_beam_select(logits, score, beams, finished=finished, eos=end)
        comet.comet_beam_reorder([history, cache[:, :, :step + 1]], parent)
        history[:, :, step] = token
        finished = finished.gather(1, parent.long()) | (token == end)
        last = token.long()
    return score, history


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--vocabulary", type=int, default=4001)
    ap.add_argument("--kept", type=int, default=32)
    ap.add_argument("--rank", type=int, default=32)
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--length", type=int, default=12)
    a = ap.parse_args(argv)
    generator = torch.Generator(device="cuda")
    generator.manual_seed(0)
    table, out, first, last = train(a.vocabulary, a.kept, a.rank, a.steps, generator)
    print("loss: %.3f over the first ten steps, %.3f over the last ten" % (first, last))
    prompts = torch.arange(2, 6, device="cuda")
    score, tokens = search(table, out, prompts, a.beams, a.length, end=0)
    greedy, _ = search(table, out, prompts, 1, a.length, end=0)
    for b in range(prompts.numel()):
        print("prompt %d: log probability %.3f (one beam: %.3f), tokens %s" % (
            int(prompts[b]), float(score[b, 0]), float(greedy[b, 0]), tokens[b, 0].tolist()))
    return first, last, score, greedy


if __name__ == "__main__":
    main()
