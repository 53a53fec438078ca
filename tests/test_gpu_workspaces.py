"""Workspaces of a context whose calls are recorded into graphs, dealt to many streams, handed back."""
import pytest
import torch

pytestmark = pytest.mark.gpu

CODE = dict(m=4, prim_poly=0x13, n=12, k=8, fcr=1)
GROUPS, BITS = 8, 48


@pytest.fixture(scope="module")
def qrm():
    import paper_2509_02447_amd as q
    return q


@pytest.fixture()
def ctx(qrm):
    c = qrm.Context(rs=CODE)
    yield c
    c.close()


class Step:
    """A norm in two launches with its backward pass and a loss of several workgroups, on inputs of its own."""

    def __init__(self, qrm, ctx, seed, n=3, p=9000, c=64, images=6000):
        g = torch.Generator().manual_seed(seed)
        self.ctx, self.images = ctx, images
        self.x, self.dy = (torch.randn((n, p, c), generator=g).cuda() for _ in range(2))
        self.logits, self.target = torch.randn((images, BITS), generator=g).cuda(), torch.randint(0, 2, (BITS,), generator=g, dtype=torch.uint8).cuda()
        self.desc = qrm.group_norm_desc(n, p, c, GROUPS, torch.float32, "silu")
        self.out = [torch.empty_like(self.x), torch.empty((n, GROUPS), device="cuda"), torch.empty((n, GROUPS), device="cuda"), torch.empty_like(self.x),
                    torch.empty(c, device="cuda"), torch.empty(1, device="cuda"), torch.empty_like(self.logits)]

    def __call__(self):
        y, mean, rstd, dx, dgamma, loss, dz = self.out
        self.ctx.qrm_group_norm(self.desc, self.x, None, None, y, mean, rstd)
        self.ctx.qrm_group_norm_backward(self.desc, self.x, self.dy, None, None, mean, rstd, dx, dgamma)
        self.ctx.qrm_message_loss(self.logits, self.target, 1, self.images, BITS, 1.0, loss, dz)

    def expect(self):
        self()
        torch.cuda.synchronize()
        self.want = [t.clone() for t in self.out]

    def check(self):
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(self.out, self.want))
        for t in self.out:
            t.fill_(5.0)
        torch.cuda.synchronize()


def record(call, stream):
    """call() on the stream, then once more into a graph."""
    with torch.cuda.stream(stream):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    return graph


def test_what_a_recorded_call_works_in_stays_when_a_larger_call_follows(qrm, ctx):
    small, large, larger = Step(qrm, ctx, 1), Step(qrm, ctx, 2, n=7, p=20000, c=128), Step(qrm, ctx, 3, n=9, p=20000, c=192)
    for s in (small, large, larger):
        s.expect()
    stream = torch.cuda.Stream()
    graph = record(small, stream)
    at, size, kept = ctx.qrm_diag_workspace(stream)
    assert at and kept == 0
    with torch.cuda.stream(stream):
        large()
    torch.cuda.synchronize()
    now, more, kept = ctx.qrm_diag_workspace(stream)
    assert more > size and now != at and kept == 1            # (the second call had to have other memory)
    large.check()
    for _ in range(3):
        with torch.cuda.stream(stream):
            graph.replay()
            large()
        small.check(), large.check()
    with torch.cuda.stream(stream):
        larger()
    larger.check()
    assert ctx.qrm_diag_workspace(stream)[2] == 1             # (no graph has seen the second)
    second = record(large, stream)
    assert ctx.qrm_diag_workspace(stream)[2] == 1
    for _ in range(3):
        with torch.cuda.stream(stream):
            graph.replay(), second.replay()
        small.check(), large.check()
    ctx.qrm_release_stream(stream)
    assert ctx.qrm_diag_workspace(stream) == (None, 0, 0)
    with torch.cuda.stream(stream):                          # a stream as any other again
        small(), large()
    small.check(), large.check()


def test_a_graphs_workspace_serves_no_other_stream(qrm, ctx):
    """Two streams with graphs, and more others than workspaces, twice over; replays between them, waited for by nobody."""
    steps = [Step(qrm, ctx, 10 + i) for i in range(4)]
    for s in steps:
        s.expect()
    streams = [torch.cuda.Stream() for _ in range(2 * qrm.QRM_MAX_STREAMS + 5)]
    own, others = streams[:2], streams[2:]
    graphs = [record(s, t) for s, t in zip(steps, own)]
    at = [ctx.qrm_diag_workspace(t)[0] for t in own]
    assert all(at) and at[0] != at[1]
    for i in range(2 * len(others)):
        for g, t in zip(graphs, own):
            with torch.cuda.stream(t):
                g.replay()
        with torch.cuda.stream(others[i % len(others)]):
            steps[2 + i % 2]()
        assert ctx.qrm_diag_workspace(others[i % len(others)])[0] not in at
        assert [ctx.qrm_diag_workspace(t)[0] for t in own] == at
        for s in (steps[0], steps[1], steps[2 + i % 2]):
            s.check()
    for t in streams:
        ctx.qrm_release_stream(t)


def test_every_workspace_in_a_graph(qrm, ctx):
    """Graphs on more streams than there are workspaces, then calls on further ones."""
    streams = [torch.cuda.Stream() for _ in range(qrm.QRM_MAX_STREAMS + 6)]
    steps = [Step(qrm, ctx, 20 + i, p=3000, images=5000) for i in range(len(streams))]
    for s in steps:
        s.expect()
    count = qrm.QRM_MAX_STREAMS + 3
    graphs = [record(steps[i], streams[i]) for i in range(count)]
    at = [ctx.qrm_diag_workspace(streams[i])[0] for i in range(count)]
    assert len(set(at)) == count
    for s in steps:
        s.check()
    for _ in range(2):
        for i, t in enumerate(streams):
            with torch.cuda.stream(t):
                graphs[i].replay() if i < count else steps[i]()
        for s in steps:
            s.check()
    assert len(set(at) | {ctx.qrm_diag_workspace(t)[0] for t in streams[count:]}) == len(streams)


@pytest.mark.parametrize("chain", [False, True])
def test_a_recorded_detection_keeps_its_workspace(qrm, chain):
    """The same for the detector's calls, with all blocks in one launch (whose state lies beside the workspace) and without."""
    import synth
    cfg = synth.CONFIGS["C1"]
    ctx = qrm.Context(weights=synth.config_weights(cfg), rs=dict(m=cfg.m, prim_poly=cfg.prim_poly, n=cfg.n, k=cfg.k, fcr=cfg.fcr))
    ctx.qrm_diag_set_flags(qrm.binding.QRM_DIAG_CHAIN_ALWAYS if chain else qrm.binding.QRM_DIAG_NO_CHAIN)
    most = 40
    d_img, d_off = torch.from_numpy(synth.images(cfg, 0, most)).cuda(), torch.from_numpy(synth.offsets(cfg, 0, most)).cuda()

    def buffers():
        return [torch.empty((most, cfg.n_bits), device="cuda"), torch.empty((most, cfg.k), dtype=torch.uint8, device="cuda"),
                torch.empty(most, dtype=torch.int8, device="cuda")]

    def call(n, out):
        ctx.qrm_detect(d_img, n, cfg.H, cfg.W, d_off, cfg.tile, out[0], None, out[1], None, out[2])

    want, replayed, eager = buffers(), buffers(), buffers()
    call(most, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2 * qrm.QRM_MAX_STREAMS + 3)]
    graph = record(lambda: call(9, replayed), streams[0])
    at = ctx.qrm_diag_workspace(streams[0])[0]
    with torch.cuda.stream(streams[0]):
        call(most, eager)
    torch.cuda.synchronize()
    assert ctx.qrm_diag_workspace(streams[0])[2] == 1 and ctx.qrm_diag_workspace(streams[0])[0] != at
    mine = (at, ctx.qrm_diag_workspace(streams[0])[0])
    for t in streams[1:] * 2:
        with torch.cuda.stream(streams[0]):
            graph.replay()
        with torch.cuda.stream(t):
            call(most, eager)
        assert ctx.qrm_diag_workspace(t)[0] not in mine
        torch.cuda.synchronize()
        for got, n in ((replayed, 9), (eager, most)):
            assert all(torch.equal(a[:n], b[:n]) for a, b in zip(got, want))
            for a in got:
                a.zero_()
        torch.cuda.synchronize()
    ctx.qrm_release_stream(streams[0])
    ctx.close()


def test_a_workspace_is_taken_over_without_the_host_waiting(qrm):
    """Fine-tuning and detection calls on more streams than workspaces, beside a stream that is busy for long: all of them return before it is done."""
    import synth
    cfg = synth.CONFIGS["C1"]
    ctx = qrm.Context(weights=synth.config_weights(cfg), rs=dict(m=cfg.m, prim_poly=cfg.prim_poly, n=cfg.n, k=cfg.k, fcr=cfg.fcr))
    n = 16
    d_img, d_off = torch.from_numpy(synth.images(cfg, 0, n)).cuda(), torch.from_numpy(synth.offsets(cfg, 0, n)).cuda()
    logits, msg, nerr = torch.empty((n, cfg.n_bits), device="cuda"), torch.empty((n, cfg.k), dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.int8, device="cuda")
    x = torch.randn((2, 9000, 64), generator=torch.Generator().manual_seed(1)).cuda()
    y, desc = torch.empty_like(x), qrm.group_norm_desc(2, 9000, 64, GROUPS, torch.float32)

    def detect(stream):
        ctx.qrm_detect(d_img, n, cfg.H, cfg.W, d_off, cfg.tile, logits, None, msg, None, nerr, stream=stream)

    def norm(stream):
        ctx.qrm_group_norm(desc, x, None, None, y, stream=stream)

    streams = [torch.cuda.Stream() for _ in range(3 * qrm.QRM_MAX_STREAMS)]
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    b = torch.empty_like(a)
    norm(streams[0])                                         # (before there is a second stream)
    for s in streams[:qrm.QRM_MAX_STREAMS + 4]:               # all workspaces are there, and large enough
        detect(s), norm(s)
    busy, done = torch.cuda.Stream(), torch.cuda.Event()
    with torch.cuda.stream(busy):
        torch.matmul(a, a, out=b)
        torch.cuda.synchronize()
        for _ in range(200):
            torch.matmul(a, a, out=b)
        done.record()
    for s in streams[qrm.QRM_MAX_STREAMS + 4:]:
        norm(s), detect(s), norm(s)
    assert not done.query()
    torch.cuda.synchronize()
    want = torch.nn.functional.group_norm(x.double().transpose(1, 2), GROUPS, eps=1e-6).transpose(1, 2)
    assert float((y - want).abs().max()) <= 1e-5             # (values of up to 5, a few roundings of 2^-22)
    ctx.close()


def test_streams_that_are_gone_are_released(qrm, ctx):
    """A stream that is destroyed before it is handed back: alone on its context, and beside another one."""
    import ctypes
    hip = ctypes.CDLL("libamdhip64.so")
    step = Step(qrm, ctx, 40)
    step.expect()
    for beside in (False, True):
        own = qrm.Context(rs=CODE)
        step.ctx = own
        handle = ctypes.c_void_p()
        assert hip.hipStreamCreateWithFlags(ctypes.byref(handle), 1) == 0
        if beside:
            step()
            torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.ExternalStream(handle.value)):
            step()
        step.check()
        assert hip.hipStreamDestroy(handle) == 0
        assert own.qrm_diag_workspace(handle.value)[0]
        own.qrm_release_stream(handle.value)
        assert own.qrm_diag_workspace(handle.value) == (None, 0, 0)
        step()
        step.check()
        own.close()
