"""Calls on a stream that is not the current one: what they allocate (scratch, results, fills and copies of their own) belongs to their stream, so that
the current stream's tensors and theirs never meet, whatever the allocator hands out while the work is still queued."""
import pytest
import torch

from paper_2411_19460_b200 import build as ssd_build
from paper_2411_19460_b200 import libssd
from tests.test_packed import make, make_conv
from tests.test_packed_ranges import call, header, plan_of

CYCLES = 60_000_000          # about 30 ms, in which the host has queued all that follows


@pytest.fixture(scope="module", autouse=True)
def built():
    ssd_build.build()


def behind_a_pause(f, sizes):
    """f(stream) with the stream kept busy; meanwhile the current stream fills new tensors of these sizes.  Returns f's results."""
    s = torch.cuda.Stream()
    fill = lambda: [torch.full((n,), 0x5a, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]      # noqa: E731
    fill()                            # memory and kernels are there then: making and loading them waits for the device
    with torch.cuda.stream(s):
        fill()
        torch.cuda._sleep(1)
        torch.cuda.synchronize()
        torch.cuda._sleep(CYCLES)
    got = f(s)
    mine = fill()
    torch.cuda.current_stream().synchronize()
    assert not s.query(), "the pause was too short for what this test looks for"
    torch.cuda.synchronize()
    for t in mine:
        assert bool((t == 0x5a).all())
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_prompts(dtype):
    t = make([5000, 77], 2, 1, 128, dtype, seed=51)
    before = t["state"].clone()
    plan = plan_of(t)
    assert header(plan)[1] > 0
    scratch = libssd.alloc_packed_workspace(plan, t["x"], t["Bm"]).numel()
    y = call(plan, t)
    after = t["state"].clone()
    t["state"].copy_(before)
    size = y.numel() * y.element_size()
    del plan
    got = behind_a_pause(lambda s: call(plan_of(t), t, stream=s), [scratch, size, plan_of(t).host.numel()])      # the plan is dropped at once
    assert torch.equal(got, y) and torch.equal(t["state"], after)


@pytest.mark.gpu
def test_conv_of_packed_prompts_and_single_tokens():
    C = 520
    t = make_conv(200, C, "bf16", 3, seed=52)
    cu = [0, 60, 190]
    state = t["state"].clone()
    out = torch.empty(200, C, dtype=torch.bfloat16, device="cuda")
    libssd.ssd_conv_packed_fwd(libssd.PackedPlan(cu, nslots=3, heads=4), t["u"], t["w"], t["bias"], t["state"], out=out)
    after = t["state"].clone()
    t["state"].copy_(state)
    got = behind_a_pause(lambda s: libssd.ssd_conv_packed_fwd(libssd.PackedPlan(cu, nslots=3, heads=4), t["u"], t["w"], t["bias"], t["state"], stream=s),
                         [out.numel() * 2, libssd.PackedPlan(cu, nslots=3, heads=4, device="cpu").host.numel()])
    assert torch.equal(got[:190], out[:190]) and torch.equal(t["state"], after)
    u = t["u"][:3]
    ref = libssd.ssd_conv_step(u, t["w"], t["bias"], t["state"].clone())
    got = behind_a_pause(lambda s: libssd.ssd_conv_step(u, t["w"], t["bias"], t["state"], stream=s), [ref.numel() * 2])
    assert torch.equal(got, ref)
    d = make([3], 4, 1, 128, "bf16", seed=53, nslots=3)
    args = [d[k] for k in ("x", "dt", "A", "Bm", "Cm", "D")]
    ref = libssd.ssd_decode_slots(*args, d["state"].clone())
    got = behind_a_pause(lambda s: libssd.ssd_decode_slots(*args, d["state"], stream=s), [ref.numel() * 2])
    assert torch.equal(got, ref)


@pytest.mark.gpu
def test_clipping():
    g = torch.Generator().manual_seed(54)
    grads = [torch.randn(n, generator=g).cuda() for n in (300000, 17, 4096)]
    outs = [torch.empty_like(v) for v in grads]
    norm = float(libssd.ssd_grad_clip(grads, 1.0, out=outs))
    scratch = libssd.alloc_grad_clip_workspace(grads).numel()
    got = behind_a_pause(lambda s: libssd.ssd_grad_clip(grads, 1.0, stream=s), [scratch, 4])
    assert float(got) == norm and all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.gpu
def test_calls_of_the_layer():
    """Fills of gradients that are summed up, scratch and dense copies of the older calls."""
    g = torch.Generator().manual_seed(55)
    B, L, C = 1, 640, 256
    u, w, bias = torch.randn(B, L, C, generator=g).cuda(), torch.randn(C, 4, generator=g).cuda(), torch.randn(C, generator=g).cuda()
    dout = torch.randn(B, L, C, generator=g).cuda()
    ref = libssd.ssd_conv_bwd(u, w, bias, None, dout, None)
    got = behind_a_pause(lambda s: libssd.ssd_conv_bwd(u, w, bias, None, dout, None, stream=s), [v.numel() * 4 for v in ref])
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    z, gamma = torch.randn(B, L, C, generator=g).cuda(), torch.randn(C, generator=g).cuda()
    ref = libssd.ssd_gated_norm_bwd(u, z, gamma, dout)
    got = behind_a_pause(lambda s: libssd.ssd_gated_norm_bwd(u, z, gamma, dout, stream=s), [v.numel() * 4 for v in ref])
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    t = make([512], 4, 1, 128, "bf16", seed=56)
    args = [t[k].contiguous()[None] if t[k].dim() > 1 else t[k] for k in ("x", "dt", "A", "Bm", "Cm", "D")]
    ref = libssd.ssd_fwd(*args, t["state"], chunk=256, seg=256)
    got = behind_a_pause(lambda s: libssd.ssd_fwd(*args, t["state"], chunk=256, seg=256, stream=s), [v.numel() * v.element_size() for v in ref])
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    y, _, boundary = libssd.ssd_fwd_segmented(*args, t["state"], chunk=256, seg=256)
    ref = libssd.ssd_bwd_segmented(*args, boundary, y, chunk=256, seg=256)
    got = behind_a_pause(lambda s: libssd.ssd_bwd_segmented(*args, boundary, y, chunk=256, seg=256, stream=s),
                         [v.numel() * v.element_size() for v in ref.values()])
    assert all(torch.equal(got[k], ref[k]) for k in ref)
    wide = torch.randn(2, 5, 4, 64, generator=g).bfloat16().cuda()
    h = torch.zeros(2, 4, 64, 128, device="cuda")
    dt, b = torch.rand(2, 5, 4, generator=g).cuda(), torch.randn(2, 5, 1, 128, generator=g).bfloat16().cuda()
    token = lambda s, h: libssd.ssd_decode_step(wide[:, 2:3], dt[:, 2:3], t["A"], b[:, 2:3], b[:, 1:2], t["D"], h, stream=s)      # noqa: E731
    ref = token(None, h.clone())
    got = behind_a_pause(lambda s: token(s, h), [2 * 4 * 64 * 2, 2 * 4 * 4, 2 * 128 * 2])
    assert torch.equal(got, ref)


@pytest.mark.gpu
def test_memory_that_the_current_stream_still_works_on():
    """Blocks that were freed behind queued work of the current stream are not scratch or result of a call on another one, and a result that was freed is
    not the next one's place while the current stream still reads it."""
    t = make([5000], 2, 1, 128, "bf16", seed=57)
    before = t["state"].clone()
    plan = plan_of(t)
    y = call(plan, t)
    sizes = [libssd.alloc_packed_workspace(plan, t["x"], t["Bm"]).numel(), y.numel() * 2]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    held = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    copies = [torch.zeros(v.numel(), dtype=torch.uint8, device="cuda") for v in held]
    torch.cuda.synchronize()
    torch.cuda._sleep(CYCLES)
    for v, c in zip(held, copies):
        v.fill_(0x5a)
        c.copy_(v)
    v = None
    del held                                            # free, and filled and copied only when the pause is over
    t["state"].record_stream(s)
    with torch.cuda.stream(s):
        t["state"].copy_(before)
    first = call(plan, t, stream=s)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(first, y) and all(bool((c == 0x5a).all()) for c in copies)
    zeros, state = torch.zeros_like(t["x"]), before.clone()
    torch.cuda.synchronize()
    torch.cuda._sleep(CYCLES)
    read = first.clone()
    del first
    second = call(plan, dict(t, x=zeros, state=state), stream=s)
    torch.cuda.synchronize()
    assert torch.equal(read, y) and not torch.equal(second, y)


@pytest.mark.gpu
def test_a_captured_call_on_a_stream_of_its_own():
    t = make([5000, 33], 2, 1, 128, "bf16", seed=58)
    before = t["state"].clone()
    plan = plan_of(t)
    y = call(plan, t).clone()
    after = t["state"].clone()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.wait_stream(torch.cuda.current_stream())
        got = call(plan, t, stream=s)
        torch.cuda.current_stream().wait_stream(s)
    for _ in range(2):
        t["state"].copy_(before)
        graph.replay()
        assert torch.equal(got, y) and torch.equal(t["state"], after)


@pytest.mark.gpu
def test_the_default_stream_given_while_another_is_current():
    t = make([512], 4, 1, 128, "bf16", seed=59)
    args = [t[k].contiguous()[None] if t[k].dim() > 1 else t[k] for k in ("x", "dt", "A", "Bm", "Cm", "D")]
    y, _, boundary = libssd.ssd_fwd_segmented(*args, t["state"], chunk=256, seg=256)
    ref = libssd.ssd_bwd_segmented(*args, boundary, y, chunk=256, seg=256)
    grads = [torch.randn(5000, device="cuda")]
    out = [torch.empty_like(grads[0])]
    norm = float(libssd.ssd_grad_clip(grads, 1.0, out=out))
    torch.cuda.synchronize()
    default = torch.cuda.default_stream()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = libssd.ssd_bwd_segmented(*args, boundary, y, chunk=256, seg=256, stream=default)
        first = libssd.ssd_fwd(*args, t["state"], chunk=256, seg=256, stream=default)[0]
        clipped = libssd.ssd_grad_clip(grads, 1.0, stream=default)
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], ref[k]) for k in ref) and torch.equal(first, y)
    assert float(clipped) == norm and torch.equal(grads[0], out[0])
