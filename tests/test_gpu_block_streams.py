"""The stream that a call names: another than torch's current one, which is busy or idle meanwhile; and workspaces, which live until that stream is done with them."""
import pytest
import torch

from paper_2412_16112_amd import clear_block as cb
from paper_2412_16112_amd.optim import AdamW
from tests.test_gpu_block_adamw import HYPER, tensors
from tests.test_gpu_block_gated import inputs
from tests.test_gpu_block_norm_rotary import norm_inputs, rotary_inputs

pytestmark = pytest.mark.gpu


def busy(stream):
    """Some 50 ms of work on a stream."""
    with torch.cuda.stream(stream):
        a = torch.ones(4096, 4096, device="cuda")
        for _ in range(40):
            a = a @ a * 1e-4
    return a


def on(side, call):
    """call(stream=side) behind other work there and before torch's current stream goes on; what it returned."""
    side.wait_stream(torch.cuda.current_stream())
    held = busy(side)
    got = call(side.cuda_stream)
    assert not side.query()  # (still at it: the call did not wait, and did not go to the idle current stream)
    torch.cuda.current_stream().wait_stream(side)
    del held
    return got


def test_every_call_on_a_named_stream():
    x, w, b, dy = norm_inputs(2, 500, 256, torch.bfloat16, torch.bfloat16, True)
    q, k, positions, freqs = rotary_inputs(1, 4, 2, 100, 64, 64, 1, torch.bfloat16)
    gx, wg, wu, dh = inputs(300, 128, 264)
    y, stats = cb.layer_norm(x, w, b, save_stats=True)
    h, pre = cb.gated_ff(gx, wg, wu, save_pre=True)
    side = torch.cuda.Stream()
    calls = [lambda s: cb.rotary(q, k, positions, freqs, stream=s), lambda s: cb.layer_norm(x, w, b, save_stats=True, stream=s), lambda s: cb.layer_norm_backward(dy, x, w, b, stats, stream=s),
             lambda s: cb.gated_ff(gx, wg, wu, save_pre=True, stream=s), lambda s: (cb.gated_ff(gx[:3], wg, wu, stream=s),), lambda s: cb.gated_ff_backward(dh, gx, wg, wu, pre, stream=s)]
    for i, call in enumerate(calls):
        want = call(None)
        got = on(side, call)
        assert all(torch.equal(a, t) for a, t in zip(got, want)), i
        current = torch.cuda.current_stream().cuda_stream
        assert all(torch.equal(a, t) for a, t in zip(call(current), want)), i


@pytest.mark.parametrize("bits", [32, 8])
def test_optimizer_on_a_named_stream(bits):
    params, grads = tensors(torch.float32, seed=2)
    same = [p.clone() for p in params]
    one, other = AdamW(params, state_bits=bits, **HYPER), AdamW(same, state_bits=bits, **HYPER)
    side = torch.cuda.Stream()
    for _ in range(2):
        on(side, lambda s: one.step(grads, stream=s))
        other.step(grads)
    assert all(torch.equal(a, b) for a, b in zip(params, same))
    if bits == 8:
        args = one.exp_avgs[9], one.scales[9][0], one.exp_avg_sqs[9], one.scales[9][1]
        assert all(torch.equal(a, b) for a, b in zip(on(side, lambda s: cb.adamw_decode(*args, stream=s)), cb.adamw_decode(*args)))


def test_a_workspace_is_kept_until_its_stream_is_done():
    """What a backward call takes as a workspace goes back to torch when the call returns; memory of its size asked for on the current stream then must be another's."""
    x, w, b, dy = norm_inputs(2, 3000, 256, torch.bfloat16, torch.bfloat16, True)
    _, stats = cb.layer_norm(x, w, b, save_stats=True)
    gx, wg, wu, dh = inputs(300, 1000, 2056)
    _, pre = cb.gated_ff(gx, wg, wu, save_pre=True)
    side = torch.cuda.Stream()
    floats = cb.lib().clear_block_layer_norm_workspace(2, 3000, 256, 1)
    room = cb.lib().clear_block_gated_ff_workspace(300, 1000, 2056)
    for call, size in ((lambda s: cb.layer_norm_backward(dy, x, w, b, stats, stream=s), 4 * floats), (lambda s: cb.gated_ff_backward(dh, gx, wg, wu, pre, stream=s), room)):
        want = call(None)
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        held = busy(side)
        got = call(side.cuda_stream)
        others = [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(4)]
        assert not side.query()
        torch.cuda.synchronize()
        assert all(torch.equal(a, t) for a, t in zip(got, want))
        assert all(bool((t == 0xff).all()) for t in others)
        del held


def test_the_stream_of_a_capture():
    q, k, positions, freqs = rotary_inputs(1, 4, 2, 100, 64, 64, 1, torch.bfloat16)
    cb.rotary(q, k, positions, freqs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = cb.rotary(q, k, positions, freqs, stream=torch.cuda.current_stream().cuda_stream)
    for turn in range(3):
        q.neg_()
        graph.replay()
        eager = cb.rotary(q, k, positions, freqs)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), turn
