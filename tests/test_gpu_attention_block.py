"""The attention block of a decoder layer: the operators together as a training step and a rollout use them, eager, on another stream
and replayed from a graph."""
import pytest
import torch

import attention_ref as ref
import jet_inputs as ji
from jet_testlib import dev_bf16

pytestmark = pytest.mark.gpu
H, N_Q, N_KV, DIM = 512, 4, 2, 128
LENS = [100, 1, 0, 155]                                      # 256 tokens


@pytest.fixture(scope="module")
def env():
    import paper_2601_14243_amd as jet
    from paper_2601_14243_amd import attention_block as ab
    assert torch.cuda.is_available()
    g = torch.Generator().manual_seed(7)
    gam = [(1 + 0.2 * torch.randn(DIM, generator=g)).bfloat16().cuda() for _ in range(2)]
    w_qkv, w_o = dev_bf16(ji.weights((N_Q + 2 * N_KV) * DIM, H, 1)), dev_bf16(ji.weights(H, N_Q * DIM, 2))
    w = ab.AttentionWeights(w_qkv, w_o, N_Q, N_KV, *gam)
    cu = [sum(LENS[:i]) for i in range(len(LENS) + 1)]
    pos = torch.cat([torch.arange(n) for n in LENS]).int().cuda()
    return jet, ab, w, (w_qkv, w_o, *gam), ab.angle_table(1024, DIM, 1e4), torch.tensor(cu, dtype=torch.int32, device="cuda"), pos, cu


def _x(seed):
    return dev_bf16(ji.f32_to_bf16_bits(ji._rng(seed).standard_normal((sum(LENS), H)).astype("float32")))


def _reference(x, w_qkv, w_o, gq, gk, table, pos, cu):
    """The unquantized block in 64 bits."""
    qkv = (x @ w_qkv.T).view(-1, N_Q + 2 * N_KV, DIM)

    def rot(t, gamma):
        t = t / torch.sqrt((t * t).mean(dim=2, keepdim=True) + 1e-6) * gamma
        row = table[pos.long()][:, None]
        a, b, c, s = t[..., :DIM // 2], t[..., DIM // 2:], row[..., :DIM // 2], row[..., DIM // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], dim=2)

    q, k, v = rot(qkv[:, :N_Q], gq), rot(qkv[:, N_Q:N_Q + N_KV], gk), qkv[:, N_Q + N_KV:]
    rows = []
    for a, b in zip(cu[:-1], cu[1:]):
        see = ref.visible(b - a, b - a, True)
        o = [torch.softmax((q[a:b, h] @ k[a:b, h // 2].T * DIM ** -0.5).masked_fill(~see, -torch.inf), dim=1) @ v[a:b, h // 2] for h in range(N_Q)]
        rows.append(torch.cat(o, dim=1))
    return torch.cat(rows) @ w_o.T


def test_training_step_against_autograd_in_64_bits(env):
    """Forward and gradients of the whole block within what FP8 operands cost, in the 2-norm.  An E4M3 rounding is off by r = 2^-5.3 = 0.025
    of a value in the mean square.  Projections: r sqrt 2 = 0.036.  Scores of normed heads are about N(0, 1), off by 0.036 sqrt 2 = 0.05,
    which is the relative error of a probability: o is off by (0.036, 0.05) = 0.062 and y, two roundings later, by 0.072.
    Backward: do 0.036, dp 0.051, ds (0.051, 0.05, and delta's share) 0.08, dq and dk (0.08, 0.036) 0.09, through norm and rotation 0.1, two
    roundings later 0.105; dgamma as dq with the heads' 0.036.  Half as much again is left for correlations."""
    jet, ab, w, master, table, cu_t, pos, cu = env
    x, dy = _x(3), dev_bf16(ji.grads(sum(LENS), H, 4))
    y, saved = ab.forward(x, w, table, pos, cu_t)
    g = ab.backward(saved, dy, w)
    leaves = [t.cpu().double().requires_grad_() for t in (x, *master)]
    want = _reference(*leaves, table.cpu().double(), pos.cpu(), cu)
    want.backward(dy.cpu().double())
    far = lambda a, b: ((a.cpu().double() - b).norm() / b.norm()).item()
    assert far(y, want.detach()) < 0.108
    for name, leaf in zip(("dx", "dw_qkv", "dw_o", "dgamma_q", "dgamma_k"), leaves):
        assert far(g[name], leaf.grad) < 0.158, name


def test_decode_continues_what_prefill_wrote(env):
    """Prefill into a paged cache and decode the last token of each sequence: the query's attention is that of the whole forward pass."""
    jet, ab, w, master, table, cu_t, pos, cu = env
    x = _x(5)
    page, n_pages = 16, 24
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(6)).int()
    live = [i for i, n in enumerate(LENS) if n]
    pages = torch.zeros((len(live), -(-max(LENS) // page)), dtype=torch.int32)
    slots = torch.empty(sum(LENS), dtype=torch.int64)
    used = 0
    for r, i in enumerate(live):
        n = -(-LENS[i] // page)
        pages[r, :n] = order[used:used + n]
        used += n
        j = torch.arange(LENS[i])
        slots[cu[i]:cu[i + 1]] = pages[r][j // page].long() * page + j % page
    last = torch.tensor([cu[i + 1] - 1 for i in live])
    first = slots.clone()
    first[last] = -1                                         # prefill leaves the last token out
    shape = (n_pages, N_KV, page, DIM)
    y, saved = ab.forward(x, w, table, pos, cu_t)
    for fp8 in (False, True):
        kv = [torch.full(shape, 0x7F, dtype=torch.uint8, device="cuda") if fp8 else torch.full(shape, float("nan"), device="cuda").bfloat16() for _ in range(2)]
        cache = jet.KvCache(*kv, *([torch.full(shape[:3], float("nan"), device="cuda") for _ in range(2)] if fp8 else []))
        y1, _ = ab.forward(x, w, table, pos, cu_t, cache, first.cuda())
        assert torch.equal(y, y1)
        lens = torch.tensor([LENS[i] for i in live], dtype=torch.int32, device="cuda")
        args = (table, pos[last.cuda()].contiguous(), cache, slots[last].cuda(), pages.cuda(), lens)
        got = ab.decode(x[last.cuda()].contiguous(), w, *args)
        q = saved["q"][last.cuda()].contiguous()
        o = jet.attention_decode(q, cache, pages.cuda(), lens)
        assert torch.equal(got, ab._project(o, w)[1])
        want, tol = ref.decode(q.cpu(), cache.k.cpu(), cache.v.cpu(), *([cache.k_scale.cpu(), cache.v_scale.cpu()] if fp8 else [None, None]),
                               pages, lens.cpu(), DIM ** -0.5)
        ref.check(o, want, tol, "decode")
        if not fp8:                                          # the same keys and values: the two passes differ by their own roundings
            full, _, full_tol, _ = ref.packed_forward(saved["q"].cpu(), saved["k"].cpu(), saved["v"].cpu(), cu, cu, DIM ** -0.5, True)
            ref.check(o, full[last], full_tol[last], "decode against forward")
            ref.check(saved["o"][last.cuda()], full[last], full_tol[last], "forward")


def test_captured_training_step_and_decode_replay_to_the_eager_bytes(env):
    jet, ab, w, master, table, cu_t, pos, cu = env
    inputs = [(_x(20 + i), dev_bf16(ji.grads(sum(LENS), H, 30 + i))) for i in range(3)]
    x, dy = inputs[0][0].clone(), inputs[0][1].clone()
    B, page = 5, 16
    kv = [torch.randn((8, N_KV, page, DIM), device="cuda").bfloat16() for _ in range(2)]
    keep = [t.clone() for t in kv]
    cache = jet.KvCache(*kv)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    pages, lens, at = i32([[0, 1], [2, 0], [3, 4], [5, 0], [6, 7]]), i32([20, 1, 32, 16, 17]), i32([19, 0, 31, 15, 16])
    slots = torch.tensor([16 + 3, 32, 64 + 15, 80 + 15, 112], dtype=torch.int64, device="cuda")

    def run():
        y, saved = ab.forward(x, w, table, pos, cu_t)
        g = ab.backward(saved, dy, w)
        z = ab.decode(x[:B], w, table, at, cache, slots, pages, lens)
        return [y, z, cache.k, cache.v] + [g[n] for n in ("dx", "dw_qkv", "dw_o", "dgamma_q", "dgamma_k")]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        warm = [t.clone() for t in run()]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(warm, run()):                            # another stream, the same bytes
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    for rep in range(6):
        for t, src in zip((x, dy), inputs[rep % 3]):
            t.copy_(src)
        for t, src in zip(kv, keep):
            t.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t, src in zip(kv, keep):
            t.copy_(src)
        want = run()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), f"replay {rep}: output {i} differs from the eager call"
