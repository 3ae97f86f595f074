"""The rollout step's operators together: the example from the allocation to
the clipped gradient, and a step captured in a CUDA graph."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location(
        "continue_rollouts", os.path.join(ROOT, "examples", "continue_rollouts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("kw", [dict(), dict(prompts=2, G=3, prompt_len=33, steps=7, drafts=0,
                                             V=512, page=8, seed=3)])
def test_example(kw):
    o = example().main(**kw)
    assert o["status"] == 0
    going = o["J"].view(-1).bool()
    assert torch.equal(o["lens"] - o["start"], o["made"].int())
    assert (o["made"][~going] == 0).all() and (o["made"][going] >= o["steps"]).all()
    assert (o["made"] <= o["steps"] * (o["drafts"] + 1)).all()
    # The log-probabilities of generation and of scoring: hidden states rounded
    # to bf16 on both sides, after attention whose weights are (2 x 2^-8 of the
    # attention's magnitude each; times 4 for sum p |v| against |h|), through
    # the head: |dz| <= 16 x 2^-8 sum |w| |h|, and a log-probability moves by at
    # most twice the largest |dz|.
    h, w = o["hidden"].float(), o["head"].float()
    size = (h.abs() @ w.abs().t()).amax(1)
    cu = o["cu"].tolist()
    for i in range(len(o["a"])):
        if o["a"][i] != 0:
            bound = 2 * 16 * 2.0 ** -8 * float(size[cu[i]:cu[i + 1]].sum())
            assert abs(float(o["logp_seq"][i] - o["logp_old"][i])) <= bound
    assert torch.isfinite(o["dW"]).all() and torch.isfinite(o["dH"]).all()


def test_step_in_a_graph():
    """One captured step replayed with other lengths, tables and chunks."""
    from paper_2608_11368_gb300 import binding as B
    R, Hq, Hkv, D, page, width, pages, T, V = 5, 4, 2, 64, 16, 12, 80, 40, 300
    g = torch.Generator(device="cuda").manual_seed(0)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    lens, held, n_new, table = i32(R), i32(R), i32(R), i32(R, width)
    free, count, err = i32(pages), i32(1), i32(1)
    k, v = (torch.zeros((pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    q, kn, vn = (torch.zeros((T, h, D), dtype=torch.bfloat16, device="cuda")
                 for h in (Hq, Hkv, Hkv))
    p, ids = torch.zeros((T, V), device="cuda"), i32(T)
    u, ud = torch.zeros(T, device="cuda"), torch.zeros(R, device="cuda")
    ws = torch.empty(B.pair_attend_workspace_size(R, Hq, Hkv, D, B.PAIR_BF16), dtype=torch.uint8,
                     device="cuda")

    def step():
        kv, ho, cu, slots, taken = B.pair_pages_extend(lens, held, n_new, free, count, table, page,
                                                       T, dev_err=err)
        B.pair_cache_append(kn, vn, slots, k, v, dev_err=err)
        out, lse = B.pair_attend_paged(q, k, v, table, kv, cu, ws=ws, dev_err=err)
        return (kv, cu, slots, out, lse) + B.pair_verify_drafts(p, ids, cu, u, ud, dev_err=err)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            res = step()
    s.synchronize()
    err.zero_()
    rng = np.random.default_rng(1)
    for n in ([1, 1, 1, 1, 1], [0, 8, 3, 20, 0], [40, 0, 0, 0, 0], [0, 0, 0, 0, 0]):
        ln = rng.integers(0, 100, R)
        hl = -(-ln // page)
        order = rng.permutation(pages)
        tb, at = np.zeros((R, width), np.int32), 0
        for i in range(R):
            tb[i, :hl[i]] = order[at:at + hl[i]]
            at += int(hl[i])
        fr = np.concatenate([order[at:], np.zeros(at, np.int64)])
        for t, x in ((lens, ln), (held, hl), (n_new, n), (table, tb), (free, fr),
                     (count, [pages - at])):
            t.copy_(torch.from_numpy(np.asarray(x, np.int32)))
        for t in (q, kn, vn, k, v):
            t.normal_(generator=g)
        p.copy_(torch.softmax(3 * torch.randn((T, V), generator=g, device="cuda"), -1))
        ids.copy_(torch.randint(0, V, (T,), generator=g, device="cuda"))
        u.uniform_(generator=g)
        ud.uniform_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        assert B.pair_status_sync(err) == 0
        kv, cu, slots, out, lse, oid, logp, emit = [x.cpu() for x in res]
        want = rollout.pages_extend(ln, hl, n, fr, pages - at, tb, page, T)
        assert np.array_equal(kv, want["kv_len"]) and np.array_equal(cu, want["cu"])
        assert np.array_equal(slots, want["slots"]) and np.array_equal(table.cpu(), want["table"])
        f = lambda x: x.double().cpu().numpy()  # noqa: E731
        for t, sl in enumerate(want["slots"]):
            if sl >= 0:
                assert torch.equal(k[sl // page, sl % page], kn[t])
                assert torch.equal(v[sl // page, sl % page], vn[t])
        ro, rl, mag, _ = rollout.attend_paged(f(q), f(k), f(v), want["table"], want["kv_len"],
                                              want["cu"], D ** -0.5)
        # Weights and output each rounded once to bf16 (2^-8), fp32 sums of at
        # most 140 terms.
        assert (np.abs(f(out) - ro) <= 2 * 2.0 ** -8 * 1.02 * mag + 1e-30).all()
        fin = np.isfinite(rl)
        assert (np.isfinite(lse.numpy()) == fin).all()
        wv = rollout.verify_drafts(p.cpu().numpy(), ids.cpu().numpy(), want["cu"], u.cpu().numpy(),
                                   ud.cpu().numpy())
        assert np.array_equal(oid, wv["ids"]) and np.array_equal(emit, wv["n"])


def test_outputs_and_workspace_belong_to_the_given_stream():
    """With stream=, what a call makes is of that stream's memory: work that is
    still to run on the current stream, in memory freed there, does not reach
    it."""
    from paper_2608_11368_gb300 import binding as B
    dev = dict(device="cuda")
    i32 = dict(dtype=torch.int32, **dev)
    lens, n_new = torch.tensor([40, 41], **i32), torch.tensor([2, 2], **i32)
    held, cu = torch.tensor([3, 3], **i32), torch.tensor([0, 2, 4], **i32)
    table = torch.arange(6, **i32).view(2, 3)
    free, count = torch.arange(6, 10, **i32), torch.tensor([4], **i32)
    k = torch.randn(6, 16, 2, 64, **dev).bfloat16()
    q = torch.randn(4, 4, 64, **dev).bfloat16()
    p = torch.softmax(torch.randn(4, 500, **dev), 1)
    ids, u, ud = torch.zeros(4, **i32), torch.rand(4, **dev), torch.rand(2, **dev)
    kv = lens + n_new
    calls = (lambda **s: B.pair_pages_extend(lens, held, n_new, free, count, table, 16, 4, **s),
             lambda **s: B.pair_attend_paged(q, k, k, table, kv, cu, **s),
             lambda **s: B.pair_verify_drafts(p, ids, cu, u, ud, **s))
    s = torch.cuda.Stream()
    for call in calls:
        want = [x.clone() for x in call()]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        later = [torch.full_like(x, 77) for x in want]  # runs after the sleep
        del later
        got = call(stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    need = B.pair_attend_workspace_size(2, 4, 2, 64, B.PAIR_BF16)
    assert any(x["stream"] == s.cuda_stream and x["total_size"] >= need
               for x in torch.cuda.memory_snapshot())
