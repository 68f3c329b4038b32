"""Speculative decoding under penalties, biases and a grammar, with the draft half on a 4-bit copy of the head.

One block of every sequence is decoded in the order of the method: the draft logits come from the 4-bit head (Mx4Logits), are edited
(EditLogits: penalties from the history, biases, the grammar's masks) and drafts are drawn from them; the target logits come from the
model's own head in bf16, are edited with the drafts as their prefix, and the round is verified on both (VerifyLogits).  Whatever the
4-bit head gets wrong costs acceptance, not exactness: the committed tokens follow the edited target law.

There is no model here: hidden states are drawn at random around the embedding of a token that a sequence would say next.

    python examples/constrained_decode.py [--batch 4] [--vocab 32000] [--hidden 1024] [--window 8] [--block 32]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_14305_amd import binding as fb  # noqa: E402


def quantise_mx4(W):
    """W [V, d] in the OCP MX 4-bit form: codes [V, d / 2] (low nibble = even column) and scales [V, d / 32], both uint8.  The scale is the
    smallest power of two whose sevenfold reaches the largest magnitude of its 32 values, so that none is cut by more than a rounding."""
    V, d = W.shape
    X = W.float().view(V, d // 32, 32)
    mantissa, exponent = torch.frexp(X.abs().amax(2, keepdim=True))
    e = (exponent - 3 + (mantissa > 0.875).int()).clamp(-126, 127)
    halfway = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=W.device)
    code = torch.bucketize((X * torch.exp2(-e.float())).abs(), halfway) + 8 * (X < 0)
    code = code.to(torch.uint8).view(V, d // 2, 2)
    return code[:, :, 0] | (code[:, :, 1] << 4), (e + 127).to(torch.uint8).view(V, d // 32)


def allow_bits(allow):
    """Truth values [B, M, V] as the int32 words of Edits.allowed."""
    B, M, V = allow.shape
    padded = torch.zeros(B, M, (V + 31) // 32 * 32, dtype=torch.bool, device=allow.device)
    padded[:, :, :V] = allow
    weights = (1 << torch.arange(32, device=allow.device, dtype=torch.int64))
    words = (padded.view(B, M, -1, 32) * weights).sum(3)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


class ConstrainedRound:
    """The buffers of one shape; `draft` and `verify` are the two halves of a round."""

    def __init__(self, B, K, block, W):
        V, d = W.shape
        self.B, self.K, self.W = B, K, W
        self.codes, self.scales = quantise_mx4(W)
        self.step = fb.VerifyLogits(B, K, block, V)
        self.head4 = fb.Mx4Logits(B * K, d, V)
        self.edit_draft = fb.EditLogits(B, K, V, "f32")
        self.edit_target = fb.EditLogits(B, K, V, "bf16")

    def draft(self, h, edits, seed, step, temperature=1.0, **state):
        """Draft tokens [B, K] from hidden states h [B, K, d]; `edits` without a prefix."""
        raw = self.step.draft_logits
        self.head4(h.view(self.B * self.K, -1), self.codes, self.scales, out=raw.flatten(0, 1))
        self.edit_draft(raw, edits, temperature=temperature, out=raw)
        return self.step(seed, step=step, phase=fb.FEF_PHASE_DRAFT, **state)[0].clone()

    def verify(self, h, edits, seed, step, temperature=1.0, **state):
        """The round's outcome from the target's hidden states; `edits` with the drafts as prefix."""
        logits = (h.view(self.B * self.K, -1) @ self.W.t()).view(self.B, self.K, -1)
        self.edit_target(logits, edits, temperature=temperature, out=self.step.target_logits)
        return self.step(seed, step=step, phase=fb.FEF_PHASE_TARGET, **state)


def decode(B, K, block, W, hidden, history, allow, lists, seed=0, temperature=1.0):
    """Decodes one block of B sequences.  hidden(positions, target): hidden states [B, K, d] of these positions; history [B, H]: the
    prompt; allow [B, block, V]: the grammar; lists: penalties and biases for Edits.  Returns tokens [B, block], rounds, drafts accepted."""
    device, H = W.device, history.shape[1]
    r = ConstrainedRound(B, K, block, W)
    mask = torch.ones(B, block, dtype=torch.uint8, device=device)
    tokens = torch.full((B, block), -1, dtype=torch.int32, device=device)
    conf = torch.zeros(B, block, device=device)
    rounds = accepted = 0
    while bool(mask.any()):
        done = (mask == 0).sum(1)                                            # this example commits from left to right
        positions = (done[:, None] + torch.arange(K, device=device)).clamp(max=block - 1)
        slots = torch.gather(allow, 1, positions[:, :, None].expand(-1, -1, allow.shape[2]))
        text = torch.cat((history, tokens), 1)
        edits = dict(history=text, history_len=(H + done).int(), prompt_len=torch.full((B,), H, dtype=torch.int32, device=device),
                     allowed=allow_bits(slots), **lists)
        state = dict(mask_in=mask, conf=conf, tokens_state=tokens, final_pass=True)
        drafts = r.draft(hidden(positions, False), fb.Edits(**edits), seed, rounds, temperature, mask_in=mask)
        _, accept_len, remask = r.verify(hidden(positions, True), fb.Edits(prefix=drafts, **edits), seed, rounds, temperature, **state)
        accepted += int(accept_len.sum())
        mask.copy_(remask)
        rounds += 1
    return tokens, rounds, accepted


def main(argv=None):
    p = argparse.ArgumentParser()
    for name, value in (("batch", 4), ("vocab", 32000), ("hidden", 1024), ("window", 8), ("block", 32)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args(argv)
    B, V, d, K, block = a.batch, a.vocab, a.hidden, a.window, a.block
    g = torch.Generator(device="cuda").manual_seed(0)
    W = (torch.randn(V, d, generator=g, device="cuda") * 0.02).bfloat16()
    says = torch.randint(0, V, (B, block), generator=g, device="cuda")       # what the model leans towards at each position
    noise = torch.randn(B, block, d, generator=g, device="cuda") * (1.0 / (0.02 * d ** 0.5))

    def hidden(positions, target):
        at = positions[:, :, None].expand(-1, -1, d)
        w = W[torch.gather(says, 1, positions)].float()
        h = torch.gather(noise, 1, at) + w * (14.0 / w.square().sum(-1, keepdim=True))
        return (h if target else h * 0.97).bfloat16()

    history = torch.randint(0, V, (B, 100), generator=g, device="cuda").int()
    allow = torch.rand(B, block, V, generator=g, device="cuda") < 0.5         # a grammar that forbids half of the tokens everywhere
    lists = dict(repetition=torch.full((B,), 1.2, device="cuda"), frequency=torch.full((B,), 0.1, device="cuda"),
                 bias_ids=torch.randint(0, V, (B, 8), generator=g, device="cuda").int(), bias_values=torch.full((B, 8), -2.0, device="cuda"))
    tokens, rounds, accepted = decode(B, K, block, W, hidden, history, allow, lists)
    kept = torch.gather(allow, 2, tokens.long()[:, :, None])
    print(f"{B} sequences of {block} tokens in {rounds} rounds, {accepted} drafts accepted; "
          f"{int(kept.sum())} of {kept.numel()} tokens are what the grammar allows")
    return tokens, rounds, accepted, bool(kept.all())


if __name__ == "__main__":
    main()
