"""One iteration of an RLHF actor on the tiny decoder: transition to the generation layout, generation with several samples per
prompt over a shared paged cache, all-gather of the answers, log probabilities and a policy-gradient update, and the way back.

    python examples/rlhf_step.py

Everything between the weights and the answers that is not a plain matrix product runs in the library: hf_reshard_execute, hf_append_kv,
hf_attend, hf_token_logprobs, hf_gather_responses, hf_token_logprobs_back, hf_reshard_back.  The update touches the LM head alone.
"""
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_19256_amd import Plan, binding as B, rollout  # noqa: E402
from paper_2409_19256_amd.arena import Arena  # noqa: E402

MODEL = dict(n_layers=2, hidden=256, n_q_heads=4, n_kv_heads=4, head_dim=64, ffn=688, vocab=1024)
PROMPTS, SAMPLES, PAGE = 3, 4, 16


class Actor:
    """The decoder over the tensors of one rank's generation buffer (generation TP 1: whole matrices), with a cache per layer."""

    def __init__(self, plan, arena, rank, pages):
        self.m = m = MODEL
        self.w = {}
        for t in plan.tensors(B.HF_BUF_GEN, rank):
            x = arena.gen[t.offset // 2: t.offset // 2 + t.rows * t.cols].view(torch.bfloat16)
            self.w[B.TENSOR_NAMES[t.tensor_id], t.layer] = x.view(t.rows, t.cols) if t.rows > 1 and t.cols > 1 else x
        self.caches = [rollout.KvCache.empty(pages, m["n_kv_heads"], PAGE, m["head_dim"]) for _ in range(m["n_layers"])]
        at = torch.arange(256, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, m["head_dim"], 2, device="cuda") / m["head_dim"])
        self.cos, self.sin = at.cos().float(), at.sin().float()

    @staticmethod
    def norm(x, w):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype) * w

    def hidden(self, tokens, positions, slots, *seen):
        """Last hidden state of one token per row; its keys and values go to `slots`, and it attends over `seen` (hf_attend's
        lengths, tables and groups)."""
        m, w, n = self.m, self.w, len(tokens)
        x = w["embed", -1][tokens]
        for i in range(m["n_layers"]):
            y = self.norm(x, w["ln1", i])
            q, k, v = (F.linear(y, w[name, i]).view(n, -1, m["head_dim"]) for name in ("q", "k", "v"))
            q = self.caches[i].append(k, v, slots, positions, self.cos, self.sin, q=q)
            out, _ = self.caches[i].attend(q, *seen)
            x = x + F.linear(out.view(n, -1), w["o", i])
            y = self.norm(x, w["ln2", i])
            x = x + F.linear(F.silu(F.linear(y, w["gate", i])) * F.linear(y, w["up", i]), w["down", i])
        return self.norm(x, w["lnf", -1])


def pages_for(first, rows, length):
    """A table of fresh pages, numbered from `first`, for rows of `length` tokens."""
    width = -(-length // PAGE)
    return (first + torch.arange(rows * width, device="cuda", dtype=torch.int32)).view(rows, width), first + rows * width


def slot_of(table, rows, position):
    return table[rows, position // PAGE].long() * PAGE + position % PAGE


def generate(actor, prompts, steps, gen):
    """prompts [prompt, token] -> responses [sample, steps] and their log probabilities, SAMPLES of them to a prompt."""
    g, length = prompts.shape
    dev, n = prompts.device, g * SAMPLES
    prompt_pages, used = pages_for(0, g, length)
    own_pages, _ = pages_for(used, n, steps)
    # the prompts, all their tokens at once: every token is a row that sees the tokens up to itself, a causal mask by lengths
    row = torch.arange(g, device=dev).repeat_interleave(length)
    pos = torch.arange(length, device=dev).repeat(g)
    h = actor.hidden(prompts.flatten(), pos.int(), slot_of(prompt_pages, row, pos), (pos + 1).int(), prompt_pages[row].contiguous())
    h = h.view(g, length, -1)[:, -1].repeat_interleave(SAMPLES, 0)
    # the samples: every step attends over the prompt's pages once per prompt and over each sample's own
    offsets = torch.arange(0, n + 1, SAMPLES, device=dev, dtype=torch.int32)
    prefix = torch.full((g,), length, device=dev, dtype=torch.int32)
    seq = torch.arange(n, device=dev)
    tokens, logprobs = [], []
    for step in range(steps):
        logits = F.linear(h, actor.w["head", -1])
        noise = -torch.log(-torch.log(torch.rand(logits.shape, generator=gen, device=dev).clamp_(1e-20, 1 - 1e-7)))
        token = (logits.float() + noise).argmax(1)
        r = rollout.token_logprobs(logits, token, top=5)
        tokens.append(token)
        logprobs.append(r.logprob)
        at = torch.full((n,), step, device=dev)
        h = actor.hidden(token, (at + length).int(), slot_of(own_pages, seq, at), (at + 1).int(), own_pages, offsets, prefix, prompt_pages, SAMPLES)
    return torch.stack(tokens, 1), torch.stack(logprobs, 1)


def score(actor, prompts, responses):
    """Hidden states in front of every response token, in one pass over prompt and response: what training sees."""
    n, steps = responses.shape
    length = prompts.shape[1]
    tokens = torch.cat((prompts.repeat_interleave(SAMPLES, 0), responses), 1)
    total = length + steps
    table, _ = pages_for(0, n, total)
    row = torch.arange(n, device=tokens.device).repeat_interleave(total)
    pos = torch.arange(total, device=tokens.device).repeat(n)
    h = actor.hidden(tokens.flatten(), pos.int(), slot_of(table, row, pos), (pos + 1).int(), table[row].contiguous())
    return h.view(n, total, -1)[:, length - 1:-1]


def main(length=37, steps=21, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    plan = Plan(MODEL, (1, 4, 1), (1, 1), flags=B.HF_COPY_OWN)
    arena = Arena(plan)
    arena.train.copy_((0.05 * torch.randn(arena.train_elems, generator=gen, device="cuda")).bfloat16().view(torch.int16))
    for r in range(plan.n_ranks):
        for t in plan.tensors(B.HF_BUF_TRAIN, r):
            if t.replicated:
                arena.train[t.offset // 2: t.offset // 2 + t.rows * t.cols] = 0x3F80  # 1.0: the norms
    arena.execute()  # training layout -> every rank's generation buffer

    # generation: each rank's replica answers prompts of its own; the answers go round the micro-DP group
    slot = torch.zeros(plan.n_ranks, PROMPTS * SAMPLES, steps, dtype=torch.int32, device="cuda")
    prompts, sampled = [], []
    for rank in range(plan.n_ranks):
        actor = Actor(plan, arena, rank, 4096 // PAGE)
        prompts.append(torch.randint(0, MODEL["vocab"], (PROMPTS, length), generator=gen, device="cuda"))
        tokens, logprobs = generate(actor, prompts[-1], steps, gen)
        slot[rank] = tokens
        sampled.append(logprobs)
    gathered = torch.empty(plan.n_ranks * plan.micro_dp_size, *slot.shape[1:], dtype=torch.int32, device="cuda")
    plan.gather_responses(slot.data_ptr(), gathered.data_ptr(), slot[0].numel() * 4, Arena.stream_handle())

    # the update, on the batch that rank 0 now holds: advantages within each prompt's samples, a step on the LM head
    actor = Actor(plan, arena, 0, 8192 // PAGE)
    head = actor.w["head", -1]
    grad, worst, before, after = torch.zeros_like(head, dtype=torch.float32), 0.0, [], []
    batches = []
    for j, rank in enumerate(plan.micro_dp_peers(0)):
        responses = gathered[j].long()
        h = score(actor, prompts[rank], responses).reshape(-1, MODEL["hidden"])
        reward = (responses % 2 == 0).float().mean(1).view(PROMPTS, SAMPLES)  # even tokens are good
        advantage = (reward - reward.mean(1, keepdim=True)).view(-1, 1).expand(-1, steps).reshape(-1).contiguous()
        logits = F.linear(h, head).requires_grad_()
        logprob, entropy = rollout.logprobs(logits, responses.flatten())
        worst = max(worst, (logprob.view(-1, steps) - sampled[rank]).abs().max().item())
        loss = -(advantage * logprob).sum() - 0.001 * entropy.sum()
        loss.backward()
        grad += F.linear(logits.grad.t().float(), h.t().float())
        batches.append((h, responses.flatten(), advantage))
        before.append((advantage * logprob).sum())
    new_head = (head.float() - 2e-3 * grad / grad.abs().max()).to(head.dtype)
    for rank in range(plan.n_ranks):  # every replica's copy
        for t in plan.tensors(B.HF_BUF_GEN, rank):
            if t.tensor_id == B.HF_G_HEAD:
                arena.gen[t.offset // 2: t.offset // 2 + new_head.numel()] = new_head.flatten().view(torch.int16)
    for h, responses, advantage in batches:
        after.append((advantage * rollout.token_logprobs(F.linear(h, actor.w["head", -1]), responses).logprob).sum())
    old = arena.train.clone()
    arena.back()  # and into the training shards
    torch.cuda.synchronize()
    changed = (arena.train != old).sum().item()
    plan.close()
    return dict(samples=gathered.shape[0] * gathered.shape[1], worst=worst, before=sum(before).item(), after=sum(after).item(), changed=changed)


if __name__ == "__main__":
    r = main()
    print("%(samples)d answers gathered; sampled and recomputed log probabilities differ by at most %(worst).4f; sum of advantage x log "
          "probability %(before).3f -> %(after).3f; %(changed)d training weights changed" % r)
