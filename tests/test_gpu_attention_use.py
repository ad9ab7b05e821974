"""Attention as programs use it: captured into graphs, on streams, with workspaces of the caller,
as a layer with its gradients (examples/softmax_mixer.py)."""
import math
import os
import sys

import pytest
import torch

import paper_2308_15152_amd as emu
from test_gpu_attention_forward import DEV, TYPES, dev, inputs
from test_gpu_mixing_streams import busy, check as check_streams  # noqa: F401

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def calls(dtype):
    """(name, f(out, workspace), makers of results, bytes of workspace, inputs)."""
    x = dev(*inputs(2, 300, 300, 4, 2, 64, dtype))
    do = torch.randn(x[0].shape, device=DEV).to(dtype)
    like = [torch.empty_like(y) for y in x]
    kept = [torch.empty_like(x[0]), torch.empty(2, 300, 4, device=DEV)]
    emu.attention_emu_forward(*x, out=kept[0], lse=kept[1])
    yield ("backward", lambda out, ws: emu.attention_emu_backward(*x, *kept, do, out=out,
                                                                  workspace=ws),
           like, emu.attention_emu_backward_workspace(*x), [do])
    for b, t, n in ((2, 100, 100), (1, 20, 5000), (2, 400, 400)):
        y = dev(*inputs(b, t, n, 4, 2, 128, dtype))
        yield ("forward", lambda out, ws, y=y: emu.attention_emu_forward(
            *y, out=out[0], lse=out[1], workspace=ws),
            [torch.empty_like(y[0]), torch.empty(b, t, 4, device=DEV)],
            emu.attention_emu_forward_workspace(*y), y)
    for b, prefix, capacity in ((3, 0, 100), (70, 3000, 700), (2, 9000, 40)):
        q = torch.randn(b, 1, 8, 64, device=DEV).to(dtype)
        caches = [torch.randn(b, capacity, 2, 64, device=DEV).to(dtype) for _ in range(2)]
        pre = [torch.randn(1, prefix, 2, 64, device=DEV).to(dtype) for _ in range(2)]
        pre = pre if prefix else []
        lengths = torch.randint(1, capacity + 1, (b,), device=DEV).int()
        yield ("step", lambda out, ws, q=q, c=caches, m=lengths, p=pre: emu.attention_emu_step(
            q, *c, m, *p, out=out[0], workspace=ws), [torch.empty_like(q)],
            emu.attention_emu_step_workspace(q, *caches, *pre), [q, *caches])


def workspace(n, fill=255):
    return torch.full((n,), fill, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("dtype", TYPES)
def test_given_workspaces_and_results(dtype):
    """Whatever the workspace holds, and however large it is."""
    for name, f, out, n, _ in calls(dtype):
        f(out, None)
        want = [y.clone() for y in out]
        for size, fill in ((n, 255), (n + 1000, 0), (n, 127)):
            for y in out:
                y.fill_(math.nan)
            f(out, workspace(max(size, 1), fill))
            assert all(torch.equal(y, z) for y, z in zip(out, want)), name
        if n:
            with pytest.raises((ValueError, emu.SgemmEmuError)):
                f(out, workspace(n - 256))


@pytest.mark.parametrize("dtype", TYPES)
def test_graph_replays(dtype):
    """Two captures of each call, with results of their own and one workspace between them,
    replayed in turn with eager calls and other inputs between the replays."""
    for name, f, out, n, ins in calls(dtype):
        ws = workspace(max(n, 1))
        outs = [out, [torch.empty_like(y) for y in out]]
        f(out, ws)
        torch.cuda.synchronize()
        graphs = []
        for o in outs:
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1]):
                f(o, ws)
        mine = [torch.empty_like(y) for y in out]
        for i in range(4):
            ins[0].mul_(-0.75)
            f(mine, None)
            for o, graph in zip(outs, graphs):
                for y in o:
                    y.fill_(math.nan)
                if i % 2:
                    torch.cuda.synchronize()
                graph.replay()
            torch.cuda.synchronize()
            for o in outs:
                assert all(torch.equal(y, z) for y, z in zip(o, mine)), (name, i)


def test_on_a_stream(busy):  # noqa: F811
    x = dev(*inputs(2, 300, 300, 4, 2, 64, torch.bfloat16))
    cu = torch.tensor([5, 100, 100, 290], dtype=torch.int32, device=DEV)
    one = [y[:1] for y in x]
    long = dev(*inputs(1, 16, 6000, 4, 2, 64, torch.bfloat16))
    f32 = [y.float() for y in x]
    lengths = torch.tensor([300, 17], dtype=torch.int32, device=DEV)
    check_streams(busy, lambda s: emu.attention_emu_forward(*x, stream=s))
    check_streams(busy, lambda s: emu.attention_emu_forward(*long, stream=s))
    newest = x[0][:, :1].contiguous()
    check_streams(busy, lambda s: [emu.attention_emu_step(
        newest, x[1], x[2], lengths, long[1], long[2], stream=s)])
    for y in (x, f32):
        o, lse = emu.attention_emu_forward(*y)
        check_streams(busy, lambda s: emu.attention_emu_backward(*y, o, lse, o, stream=s))
    o, lse = emu.attention_emu_forward(*one)
    check_streams(busy, lambda s: emu.attention_emu_backward(*one, o, lse, o, cu_seqlens=cu,
                                                             stream=s))


def test_two_calls_at_once():
    """On two streams, each with what it allocates."""
    x = dev(*inputs(1, 64, 6000, 8, 2, 128, torch.bfloat16))
    want = [y.clone() for y in emu.attention_emu_forward(*x)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(emu.attention_emu_forward(*x))
    torch.cuda.synchronize()
    assert all(torch.equal(y, z) for r in got for y, z in zip(r, want))


def test_layer_and_its_gradients():
    """The example runs, and its gradients are the formulas': in FP32, where with errors of
    2^-22 relative in each of the products, sums of up to 1152 terms and factors of order
    one between them the whole is off by less than 1e-4 of the largest."""
    import softmax_mixer
    losses, off = softmax_mixer.run()
    assert all(math.isfinite(y) for y in losses)
    # the projections of one token and of many may round differently, and a bfloat16 q, k or
    # v on the edge goes to its neighbour: 2^-8 of an element, with the output's twice
    assert off < 2.0 ** -7

    torch.manual_seed(1)
    mixer = softmax_mixer.SoftmaxMixer(48, 4, 2, 32, 256, DEV, torch.float32)
    x = torch.randn(2, 90, 48, device=DEV, requires_grad=True)
    at = torch.arange(90, dtype=torch.int32, device=DEV).expand(2, -1).contiguous()
    w = torch.randn(2, 90, 48, device=DEV)
    (mixer(x, at) * w).sum().backward()

    into, out = (y.weight.detach().cpu().double().requires_grad_() for y in (mixer.into, mixer.out))
    z = x.detach().cpu().double().requires_grad_()
    q, k, v = (y.unflatten(-1, (-1, 32)) for y in (z @ into.T).split(mixer.parts, -1))
    cos, sin = (y[:90, None].cpu().double() for y in (mixer.cos, mixer.sin))

    def turned(y):
        a, b = y[..., :16], y[..., 16:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    q, k = turned(q).transpose(1, 2), turned(k).transpose(1, 2).repeat_interleave(2, 1)
    s = q @ k.mT * 32 ** -0.5
    s = s.masked_fill(torch.ones(90, 90, dtype=torch.bool).triu(1), -math.inf)
    o = (s.softmax(-1) @ v.transpose(1, 2).repeat_interleave(2, 1)).transpose(1, 2).flatten(2)
    ((o @ out.T) * w.cpu().double()).sum().backward()
    for got, want in ((mixer.into.weight.grad, into.grad), (mixer.out.weight.grad, out.grad),
                      (x.grad, z.grad)):
        assert (got.cpu().double() - want).abs().max() < 1e-4 * want.abs().max()


def test_packed_layer_is_each_sequence_by_itself():
    import softmax_mixer
    torch.manual_seed(2)
    mixer = softmax_mixer.SoftmaxMixer(48, 4, 2, 32, 256, DEV, torch.float32)
    lengths = [70, 1, 33]
    x = torch.randn(1, sum(lengths), 48, device=DEV)
    at = torch.cat([torch.arange(n) for n in lengths]).int()[None].to(DEV)
    cu = torch.tensor([0, 70, 71, 104], dtype=torch.int32, device=DEV)
    got = mixer(x, at, cu)
    for a, b in zip(cu.tolist(), cu.tolist()[1:]):
        want = mixer(x[:, a:b], at[:, a:b].contiguous())
        assert (got[:, a:b] - want).abs().max() < 1e-5 * want.abs().max() + 1e-6
