"""Steps with fewer rows than new tokens: every row that there is gives what one pass over its sequence gives,
and the tokens left out are the next step's."""
import random

import pytest

from oracle import seq
from tests.test_gpu_chunk import _i32, _serving
from tests.test_gpu_sequence import DT, _ca, _gen, _rand, _torch, _u

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,tokens", [(1, 3), (5, 40), (300, 77), (70, 2500), (1100, 3000)])
def test_lengths_as_far_as_the_rows_go(B, tokens):
    """Both growing kernels, lengths that make no sense among them."""
    import torch
    ca = _ca()
    r = random.Random(B)
    page, width = 8, 12
    pages = B * width
    for _ in range(6):
        lens = [r.randrange(-3, page * width + 20) for _ in range(B)]
        new = [r.choice((0, 1, r.randrange(-2, 120))) for _ in range(B)]
        pool, table = ca.page_pool(pages, page), torch.full((B, width), -1, dtype=torch.int32, device="cuda")
        seen = _i32([-9] * B)
        plan = ca.cache_grow(pool, table, _i32(lens), _i32(new), tokens, seen=seen)
        rows, free = [[-1] * width for _ in range(B)], list(range(pages - 1, -1, -1))
        state, starts, slots, positions = seq.cache_grow(rows, free, lens, new, page, pages, tokens)
        assert pool.state.tolist() == state and table.tolist() == rows
        assert plan.starts.tolist() == starts and plan.slots.tolist() == slots and plan.positions[0].tolist() == positions
        assert seen.tolist() == seq.lens_with_rows(lens, new, page * width, tokens)
        again = ca.cache_grow(pool, table, _i32(lens), _i32(new), tokens)
        assert all(torch.equal(a, b) for a, b in zip(plan, again))


def test_seen_refusals():
    import torch
    ca = _ca()
    pool, table, n = ca.page_pool(9, 16), _i32([[-1] * 3] * 2), _i32([5, 5])
    for seen in (torch.zeros(2, dtype=torch.int64, device="cuda"), _i32([0]), _i32([0] * 4)[::2], n, torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError, match="seen|on cuda"):
            ca.cache_grow(pool, table, n, _i32([1, 1]), 4, seen=seen)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("captured", [False, True])
def test_steps_with_fewer_rows_than_tokens(dt, captured):
    """Four prompts through arrays of 50 rows, in steps that are the same whatever fits (one graph, if captured), on a pool that
    held NaN, against one causal pass each."""
    import torch
    ca = _ca()
    g = _gen(70)
    B, n, H, Hk, d, page, T = 4, [90, 1, 133, 47], 4, 2, 64, 16, 50
    w = ca.Window(causal=True)
    s = _serving(dt, w, page, 40, B, 10, T)
    s["kp"].fill_(float("nan"))
    s["vp"].fill_(float("nan"))
    s["seen"] = _i32([0] * B)
    xs = [[_rand(g, (m, h, d), dt).cuda() for h in (H, Hk, Hk)] for m in n]
    whole = []
    for (q, k, v), m in zip(xs, n):
        qr, kr = ca.rope(s["rope"], q[None], k[None], grid=(m,), layout="bnhd")
        whole.append(ca.window_attn(w, qr, kr, v[None], layout="bnhd", want_lse=True))

    def step():
        plan = ca.cache_grow(s["pool"], s["table"], s["lens"], s["new"], T, seen=s["seen"])
        q, k = ca.rope(s["rope"], s["q"][None], s["k"][None], positions=plan.positions, layout="bnhd")
        ca.cache_write(k[0], s["v"], s["kp"], s["vp"], plan.slots)
        out, lse = ca.paged_chunk_attn(w, q[0], s["kp"], s["vp"], s["table"], s["seen"], plan.starts, want_lse=True)
        return out, lse, plan

    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()  # (no new tokens yet)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = step()
        torch.cuda.synchronize()
    at, steps = [0] * B, 0
    while at != n:
        new, rows = [m - a for a, m in zip(at, n)], 0
        for b in range(B):  # (the program packs as much as there is room for)
            m = min(new[b], T - rows)
            for x, name in zip(xs[b], ("q", "k", "v")):
                s[name][rows:rows + m] = x[at[b]:at[b] + m]
            rows += m
        s["lens"].copy_(_i32(n))
        s["new"].copy_(_i32(new))
        if captured:
            graph.replay()
            out, lse, plan = held
        else:
            out, lse, plan = step()
        assert s["pool"].state[1:].tolist() == [0, max(0, sum(new) - T)]
        seen = s["seen"].tolist()
        for b in range(B):
            i0, i1 = plan.starts[b:b + 2].tolist()
            if i0 == i1:
                continue
            want, lw = whole[b][0][0, at[b]:seen[b]].float(), whole[b][1][0, :, at[b]:seen[b]].T
            # (each within u of the exact result, relative to the values, and their own roundings)
            assert (out[i0:i1].float() - want).abs().max() <= 4 * (_u(dt) + 2.0 ** -20) * xs[b][2].float().abs().max()
            assert (lse[i0:i1] - lw).abs().max() <= 1e-4
        assert sum(seen) - sum(at) == min(T, sum(new))
        at, steps = seen, steps + 1
    assert steps == -(-sum(n) // T)
