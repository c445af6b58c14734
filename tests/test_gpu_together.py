"""The calls as a model with an image or video encoder makes them: training a cross
attention over rotated tokens, and several answers decoded over one long prompt
(MI355X). Every stage is checked in 64 bits on what the stage before it returned."""
import math

import pytest
import torch

from paper_2607_12789_amd import avq
from tests.cross_reference import check_backward, check_forward
from tests.serving_reference import check_attention, check_prompt, read_cache
from tests.test_gpu_rotate import check as check_rotated

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def cu(lens):
    return torch.tensor([0] + list(lens)).cumsum(0).int()


def tables(n_pos, half):
    a = torch.arange(n_pos).double()[:, None] * 10000.0 ** (-torch.arange(half).double() / half)
    return a.cos().float(), a.sin().float()


def grid(frames, height, width):
    """Positions (time, height, width) of a clip's patches."""
    t, y, x = torch.meshgrid(*(torch.arange(n) for n in (frames, height, width)), indexing="ij")
    return torch.stack((t, y, x), -1).view(-1, 3).int()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_training_step(dtype):
    """Text queries over the patches of two clips: rotation, attention, gradients of
    the rows before the rotation."""
    g = torch.Generator().manual_seed(0)
    Hq, Hkv, d, axis = 4, 2, 64, (0,) * 8 + (1,) * 12 + (2,) * 12
    clips = [grid(2, 5, 7), grid(1, 9, 4)]
    lens_q, lens_k, scale = [37, 5], [len(c) for c in clips], 1 / math.sqrt(d)
    q0 = torch.randn(42, Hq, d, generator=g).to(dtype)
    k0, V = (torch.randn(sum(lens_k), Hkv, d, generator=g).to(dtype) for _ in "kv")
    dY = torch.randn(42, Hq, d, generator=g).to(dtype)
    mask = torch.rand(sum(lens_k), generator=g) < 0.9
    cos, sin = tables(64, 32)
    pos_q = torch.arange(42).int()[:, None].expand(42, 3).contiguous()  # text: one position
    pos_k = torch.cat(clips)
    c = [x.cuda() for x in (cos, sin)]
    Q = avq.rotate_axes(q0.cuda(), None, pos_q.cuda(), *c, axis)[0]
    K = avq.rotate_axes(k0.cuda(), None, pos_k.cuda(), *c, axis)[0]
    check_rotated(Q, q0, pos_q, cos, sin, axis, False, False)
    check_rotated(K, k0, pos_k, cos, sin, axis, False, False)
    lens = [cu(lens_q).cuda(), cu(lens_k).cuda()]
    Y, lse = avq.cross_attention_fwd(Q, K, V.cuda(), *lens, scale, mask=mask.cuda(), with_lse=True)
    check_forward(Y.cpu(), lse.cpu(), Q.cpu(), K.cpu(), V, lens_q, lens_k, scale, mask)
    if dtype == F32:  # Y and lse are then as near to the exact ones as the bounds take them
        dQ, dK, dV = avq.cross_attention_bwd(dY.cuda(), Q, K, V.cuda(), Y, lse, *lens, scale,
                                             mask=mask.cuda())
    else:
        from tests.cross_reference import forward64
        y64, l64 = forward64(Q.cpu(), K.cpu(), V, lens_q, lens_k, scale, mask)
        dQ, dK, dV = avq.cross_attention_bwd(dY.cuda(), Q, K, V.cuda(), y64.to(dtype).cuda(),
                                             l64.float().cuda(), *lens, scale, mask=mask.cuda())
    check_backward([x.cpu() for x in (dQ, dK, dV)], dY, Q.cpu(), K.cpu(), V, lens_q, lens_k, scale,
                   mask)
    dq0 = avq.rotate_axes(dQ, None, pos_q.cuda(), *c, axis, inverse=True)[0]
    dk0 = avq.rotate_axes(dK, None, pos_k.cuda(), *c, axis, inverse=True, Q_out=dK.clone())[0]
    check_rotated(dq0, dQ.cpu(), pos_q, cos, sin, axis, False, True)
    check_rotated(dk0, dK.cpu(), pos_k, cos, sin, axis, False, True)


@pytest.mark.parametrize("fp4", [False, True])
def test_answers_to_one_clip(fp4):
    """A clip's patches are the prompt; five answers share its pages and grow by single
    tokens, which also read the states of another encoder."""
    g = torch.Generator().manual_seed(1)
    Hq, Hkv, d, ps, n = 8, 2, 64, 16, 5
    axis = tuple(i % 3 for i in range(32))
    pos = grid(3, 6, 11)  # 198 patches: 12 pages and 6 positions
    T, scale = len(pos), 1 / math.sqrt(d)
    cos, sin = tables(256, 32)
    c = [x.cuda() for x in (cos, sin)]
    E = avq.cache_page_bytes(BF16, ps, d, fp4)
    whole = T // ps
    cache = torch.zeros(whole + 3 * n, Hkv, E, dtype=torch.uint8, device="cuda")
    table = torch.zeros(n, 40, dtype=torch.int32)  # room for 640 positions
    table[:, :whole] = torch.arange(whole)
    for i in range(n):
        table[i, whole:whole + 3] = whole + 3 * i + torch.arange(3)
    dev_table = table.cuda()
    Q, K, V = (torch.randn(T, h, d, generator=g).to(BF16).cuda() for h in (Hq, Hkv, Hkv))
    Q, K = avq.rotate_axes(Q, K, pos.cuda(), *c, axis)
    avq.cache_append(K, V, cache, dev_table[:1], torch.zeros(1, dtype=torch.int32, device="cuda"), ps,
                     cu=cu([T]).cuda(), fp4=fp4)
    Y, lse = avq.prompt_attention_fwd(Q, K, V, cu([T]).cuda(), cu([T]).cuda(), scale, causal=False,
                                      with_lse=True)
    check_prompt(Y.cpu(), lse.cpu(), Q.cpu(), K.cpu(), V.cpu(), [T], [T], scale, False)
    # the page in which the prompt ends: a copy for each answer
    for i in range(1, n):
        cache[table[i, whole]] = cache[table[0, whole]]
    lens = torch.full((n,), T, dtype=torch.int32, device="cuda")
    groups = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n], [T])]
    states = [torch.randn(90, Hkv, d, generator=g).to(BF16).cuda() for _ in "kv"]
    seen = torch.rand(90, generator=g) < 0.8
    for step in range(12):
        q, k, v = (torch.randn(n, h, d, generator=g).to(BF16).cuda() for h in (Hq, Hkv, Hkv))
        at = torch.full((n, 3), 11 + step, dtype=torch.int32, device="cuda")
        q, k = avq.rotate_axes(q, k, at, *c, axis)
        avq.cache_append(k, v, cache, dev_table, lens, ps, fp4=fp4)
        lens = lens + 1
        y, lse = avq.cache_prefix_attention_fwd(q[:, None], cache, dev_table, lens, *groups, ps, scale,
                                                fp4=fp4, with_lse=True)
        for i in range(n):
            K64, V64, _ = read_cache(cache.cpu(), table, i, T + step + 1, BF16, fp4, ps, d)
            for h in range(Hq):
                check_attention(y[i, :, h].cpu(), lse[i, :, h].cpu(), q[i, h][None].cpu(),
                                K64[h // 4], V64[h // 4], scale, torch.tensor([T + step + 1]),
                                f"step {step} answer {i} head {h}")
        # all answers read one source: its queries are simply packed together
        y, lse = avq.cross_attention_fwd(q, *states, cu([n]).cuda(), cu([90]).cuda(), scale,
                                         mask=seen.cuda(), with_lse=True)
        check_forward(y.cpu(), lse.cpu(), q.cpu(), states[0].cpu(), states[1].cpu(), [n], [90], scale,
                      seen)
