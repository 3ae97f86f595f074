"""From the allocation of a step to its clipped gradient, with the rollouts
generated in between, on one GPU:

    pair_allocate        continuation probabilities, from which J is drawn;
    pair_pages_extend,   every step: pages and slots for the continued
    pair_cache_append,   rollouts' chunks (the last token and its drafts),
    pair_attend_paged,   their keys and values, attention over the cache,
    pair_verify_drafts   and the drafts against the target's probabilities;
    pair_coeffs_product  coefficients of the completed rollouts;
    pair_attend_paged    the hidden states of whole rollouts in one chunk each;
    pair_grad_clipped    the surrogate, with the log-probabilities that the
                         verification returned as the old ones.

The policy is a random single attention layer with an output head; the drafter
is the head applied to the embedding of the last token. Run it with
    python examples/continue_rollouts.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_11368_gb300 import binding as B  # noqa: E402


class Policy:
    """One attention layer: hidden state of a token = its attention output."""

    def __init__(self, V, Hq, Hkv, D, g):
        def w(*shape):
            x = torch.randn(shape, generator=g, device="cuda") * shape[-1] ** -0.5
            return x.bfloat16()

        d = Hq * D
        self.V, self.Hq, self.Hkv, self.D, self.d = V, Hq, Hkv, D, d
        self.embed = torch.randn((V, d), generator=g, device="cuda").bfloat16()
        self.wq, self.wkv, self.head = w(d, d), w(2 * Hkv * D, d), w(V, d)

    def qkv(self, ids):
        x = self.embed[ids.long()]
        kv = (x @ self.wkv.t()).view(-1, 2, self.Hkv, self.D)
        return (x @ self.wq.t()).view(-1, self.Hq, self.D), kv[:, 0], kv[:, 1]

    def probs(self, hidden, sharp=8.0):
        return torch.softmax(sharp * (hidden.float() @ self.head.float().t()), -1)


class Cache:
    """Pages of all requests and the list of free ones, on the device."""

    def __init__(self, policy, R, pages, page, width):
        shape = (pages, page, policy.Hkv, policy.D)
        self.k, self.v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in "kv")
        self.page = page
        self.table = torch.zeros((R, width), dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.held = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, device="cuda").to(torch.int32)
        self.count = torch.full((1,), pages, dtype=torch.int32, device="cuda")
        self.at = torch.arange(pages, device="cuda")

    def extend(self, n_new, T, err):
        """Pages and slots for n_new tokens per request; the table, the pages
        held and the free list move on, lens stays until tokens are accepted."""
        kv_len, self.held, cu, slots, taken = B.pair_pages_extend(
            self.lens, self.held, n_new, self.free, self.count, self.table, self.page, T,
            dev_err=err)
        self.free = self.free[(self.at + taken).clamp_max(len(self.at) - 1)]
        self.count = self.count - taken
        return kv_len, cu, slots


def chunk(policy, cache, ids, n_new, T, err, max_new=0):
    """Hidden states [T, d] of a chunk of tokens per request, which go into the
    cache; and the chunks' offsets."""
    kv_len, cu, slots = cache.extend(n_new, T, err)
    q, k, v = policy.qkv(ids)
    B.pair_cache_append(k, v, slots, cache.k, cache.v, dev_err=err)
    out, _ = B.pair_attend_paged(q, cache.k, cache.v, cache.table, kv_len, cu, max_new=max_new,
                                 dev_err=err)
    return out.view(T, policy.d), cu


def main(prompts=4, G=8, prompt_len=100, steps=24, drafts=3, V=4096, page=16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    policy = Policy(V, 4, 2, 128, g)
    R, n = prompts * G, drafts + 1
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    longest = prompt_len + steps * n
    cache = Cache(policy, R, R * (longest // page + 2), page, longest // page + 2)

    # Which rollouts go on: the design's probabilities, and the draw.
    p_hat = 0.05 + 0.9 * torch.rand((prompts, G), generator=g, device="cuda")
    cost = 0.5 + torch.rand((prompts, G), generator=g, device="cuda")
    pi, _ = B.pair_allocate(cost, 0.6 * cost.sum(1), 0.08, p_hat=p_hat, dev_err=err)
    J = (torch.rand((prompts, G), generator=g, device="cuda") < pi).to(torch.uint8)
    go = J.view(R).to(torch.int32)

    # Prompts without their last token, which the first step takes: a group's
    # rollouts share the pages that they fill, written by its first one; the rest of
    # the prompt is each rollout's own chunk.
    prompt = torch.randint(0, V, (prompts, prompt_len), generator=g, device="cuda")
    full = (prompt_len - 1) // page * page
    first = torch.zeros(R, dtype=torch.int32, device="cuda")
    first[::G] = full
    if full:
        chunk(policy, cache, prompt[:, :full].reshape(-1), first, prompts * full, err, full)
        cache.table.view(prompts, G, -1)[:, 1:, :full // page] = \
            cache.table.view(prompts, G, -1)[:, :1, :full // page]
        cache.lens += full
        cache.held += full // page - (cache.held > 0).int() * (full // page)
    rest = torch.full((R,), prompt_len - 1 - full, dtype=torch.int32, device="cuda")
    own = prompt[:, full:-1].repeat_interleave(G, 0)
    if prompt_len - 1 > full:
        chunk(policy, cache, own.reshape(-1), rest, R * (prompt_len - 1 - full), err)
        cache.lens += rest
    last = prompt[:, -1].repeat_interleave(G).to(torch.int32)
    start = cache.lens.clone()

    # Steps. A stopped rollout has an empty chunk; T rows are enough for all.
    T = R * n
    ids_all = torch.full((R, steps * n + 1), -1, dtype=torch.int32, device="cuda")
    ids_all[:, 0] = last
    made = torch.zeros(R, dtype=torch.int64, device="cuda")
    logp_all = torch.zeros((R, steps * n + 1), device="cuda")
    lane = torch.arange(n, device="cuda")
    for _ in range(steps):
        # Drafts, one after the other, from the drafter's probabilities.
        q = torch.empty((R, n, V), device="cuda")
        toks = [last]
        for j in range(drafts):
            q[:, j] = policy.probs(policy.embed[toks[-1].long()], 0.1)
            toks.append(torch.multinomial(q[:, j], 1, generator=g)[:, 0].to(torch.int32))
        toks = torch.stack(toks, 1)
        # The packed rows: the continued requests' chunks, then spare rows.
        order = torch.argsort(1 - go, stable=True)
        ids = toks[order].reshape(-1).contiguous()
        hidden, cu = chunk(policy, cache, ids, go * n, T, err, n)
        out, logp, emit = B.pair_verify_drafts(
            policy.probs(hidden), ids, cu, torch.rand(T, generator=g, device="cuda"),
            torch.rand(R, generator=g, device="cuda"), q=q[order].view(T, V), dev_err=err)
        # Bookkeeping per request: tokens, log-probabilities, cache lengths.
        back = torch.argsort(order)
        out, logp = out.view(R, n)[back], logp.view(R, n)[back]
        new = lane < emit[:, None]
        where = torch.where(new, made[:, None] + 1 + lane, 0)
        ids_all.scatter_(1, where, torch.where(new, out, ids_all[:, :1]))
        logp_all.scatter_(1, where, torch.where(new, logp, 0.0))
        made += emit
        cache.lens = cache.lens + emit
        last = torch.where(emit > 0, out.gather(1, (emit.long() - 1).clamp_min(0)[:, None])[:, 0],
                           last)

    # Rewards stand in for a verifier's: the last token's parity.
    r = (last % 2).float().view(prompts, G)
    a, *_ = B.pair_coeffs_product(r, J, pi, scale=2.0 / (G * (G - 1)), dev_err=err)

    # The surrogate over the generated tokens: their hidden states in one chunk
    # per rollout, over the cache that the steps left.
    seq = [ids_all[i, :int(made[i]) + 1] for i in range(R)]
    cu_seq = torch.zeros(R + 1, dtype=torch.int32, device="cuda")
    cu_seq[1:] = made.cumsum(0)
    T = int(cu_seq[-1])
    ids = torch.cat([s[:-1] for s in seq])
    y = torch.cat([s[1:] for s in seq]).contiguous()
    logp_tokens = torch.cat([logp_all[i, 1:len(s)] for i, s in enumerate(seq)])
    logp_old = logp_all.sum(1)
    q, _, _ = policy.qkv(ids)
    hidden, _ = B.pair_attend_paged(q, cache.k, cache.v, cache.table, cache.lens, cu_seq,
                                    max_new=int(made.max()), dev_err=err)
    hidden = (8.0 * hidden.view(T, policy.d)).contiguous()  # the policy's sharpness
    Jobj, dH, dW, logp_seq, coef = B.pair_grad_clipped(
        hidden, policy.head, y, torch.ones(T, dtype=torch.uint8, device="cuda"), cu_seq,
        a.reshape(-1).contiguous(), logp_old, dev_err=err)
    status = B.pair_status_sync(err)
    return dict(status=status, J=J, made=made, start=start, lens=cache.lens, logp_old=logp_old,
                logp_tokens=logp_tokens, logp_seq=logp_seq, a=a.reshape(-1), coef=coef, Jobj=Jobj,
                dH=dH, dW=dW, hidden=hidden, y=y, cu=cu_seq, head=policy.head, steps=steps,
                drafts=drafts)


if __name__ == "__main__":
    o = main()
    going = o["J"].view(-1).bool()
    print("status %d, %d of %d rollouts continued, %d tokens, %.2f per step and rollout"
          % (o["status"], int(going.sum()), going.numel(), int(o["made"].sum()),
             float(o["made"][going].float().mean()) / o["steps"]))
    active = o["a"] != 0
    print("ratio to the old log-probabilities %.4f .. %.4f, J %.6f, |dW| %.4e"
          % (float((o["logp_seq"] - o["logp_old"])[active].exp().min()) if active.any() else 1.0,
             float((o["logp_seq"] - o["logp_old"])[active].exp().max()) if active.any() else 1.0,
             float(o["Jobj"]), float(o["dW"].norm())))
