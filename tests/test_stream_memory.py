"""Where a call is given a stream, what it allocates for itself and what it returns belong to that
stream: memory of the current stream may still be in use there, and whoever gets it there next
would not wait for the call's kernels.

The first test needs no GPU: it runs the binding's Python on stand-ins and looks at the stream that
every allocation was made under.  The others run the calls on a stream that is kept busy, with
allocations and writes on the current stream right behind them."""
import types

import pytest
import torch

CURRENT, GIVEN = 111, 222
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Device(torch.Tensor):
    """A host tensor that passes for one of a GPU."""
    is_cuda = True
    __torch_function__ = torch._C._disabled_torch_function_impl


class Library:
    """Every entry point succeeds and does nothing; the stream that each was given is kept."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            if not name.endswith("_workspace") and name != "sn_wire_bytes":
                self.streams.append(args[-1])
            return 0
        return call


def device(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Device)


def calls(sn):
    """Each call that allocates, as a function of the stream."""
    T, d, k, V = 4, 64, 8, 32
    b = types.SimpleNamespace(handle=1, d=d, k=k)
    grads = types.SimpleNamespace(handle=1, device=torch.device("cpu"))
    X, C, E = device(T, d), device(T, k), device(V, d)
    w, M, U = device(d, dtype=F32), device(d, k, dtype=F32), device(V, k, dtype=F32)
    ids, row, lse = device(T, dtype=I32), device(T, dtype=F32), device(T, 2, dtype=F32)
    codes, bits = device(T, d, dtype=torch.uint8), device(T, d // 32, dtype=I32)
    cols, one = device(T, k, dtype=torch.int16), device(1, dtype=torch.float64)
    W = device(d, V)
    A = [device(d, V, dtype=F32) for _ in range(4)]
    return {
        "compress_fwd": lambda s: sn.sn_compress_fwd(b, X, ids, E, T, stream=s),
        "project_tables": lambda s: sn.sn_project_tables(b, E, X, stream=s),
        "compress_fwd_projected": lambda s: sn.sn_compress_fwd_projected(b, X, ids, U, T, stream=s),
        "build_ts": lambda s: sn.sn_build_ts(b, E, stream=s),
        "grassmann_accumulate": lambda s: sn.sn_grassmann_accumulate(b, X, C, M, stream=s),
        "grassmann_step": lambda s: sn.sn_grassmann_step(b, M, 1, 0.1, stream=s),
        "adamw_rowconst": lambda s: sn.sn_adamw_rowconst(*A, 1, 0.1, stream=s),
        "topk_compress": lambda s: sn.sn_topk_compress(X, k, stream=s),
        "topk_restore": lambda s: sn.sn_topk_restore(C, cols, d, stream=s),
        "sign_compress": lambda s: sn.sn_sign_compress(X, stream=s),
        "sign_restore": lambda s: sn.sn_sign_restore(bits, row, d, stream=s),
        "quant_compress": lambda s: sn.sn_quant_compress(X, "int8", stream=s),
        "quant_restore": lambda s: sn.sn_quant_restore(codes, row, "int8", stream=s),
        "embed_fwd": lambda s: sn.sn_embed_fwd(E, ids, stream=s),
        "embed_bwd": lambda s: sn.sn_embed_bwd(X, ids, V, stream=s),
        "rmsnorm_fwd": lambda s: sn.sn_rmsnorm_fwd(X, w, 1e-5, R=X, stream=s),
        "rmsnorm_fwd_quant": lambda s: sn.sn_rmsnorm_fwd_quant(X, w, 1e-5, "int8", R=X, group=32, stream=s),
        "rmsnorm_bwd": lambda s: sn.sn_rmsnorm_bwd(X, X, w, 1e-5, stream=s),
        "logprob_fwd": lambda s: sn.sn_logprob_fwd(X, ids, top=3, stream=s),
        "logprob_bwd": lambda s: sn.sn_logprob_bwd(X, lse, ids, row, stream=s),
        "grads_sumsq": lambda s: sn.sn_grads_sumsq(grads, stream=s),
        "grads_clip": lambda s: sn.sn_grads_clip(grads, one, 1.0, stream=s),
        "decompress_fwd": lambda s: sn.sn_decompress_fwd(b, C, ids, E, T, stream=s),
        "compress_bwd": lambda s: sn.sn_compress_bwd(b, X, stream=s),
        "decompress_bwd": lambda s: sn.sn_decompress_bwd(b, C, stream=s),
        "project_weight": lambda s: sn.sn_project_weight(b, W, stream=s),
    }


NAMES = ["compress_fwd", "project_tables", "compress_fwd_projected", "build_ts", "grassmann_accumulate",
         "grassmann_step", "adamw_rowconst", "topk_compress", "topk_restore", "sign_compress", "sign_restore",
         "quant_compress", "quant_restore", "embed_fwd", "embed_bwd", "rmsnorm_fwd", "rmsnorm_fwd_quant",
         "rmsnorm_bwd", "logprob_fwd", "logprob_bwd", "grads_sumsq", "grads_clip", "decompress_fwd",
         "compress_bwd", "decompress_bwd", "project_weight"]


@pytest.fixture
def stand_in(monkeypatch):
    """The binding on host tensors: (module, streams that calls were given, allocations as pairs of
    the stream that was current and the streams that the tensor was recorded on)."""
    from paper_2506_01260_gb300 import build
    build.build()
    from paper_2506_01260_gb300 import sn
    current, made = [CURRENT], []
    library = Library()

    class Entered:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            current.append(self.stream.cuda_stream)

        def __exit__(self, *_):
            current.pop()

    def recorded(fn):
        def make(*args, **kw):
            t = fn(*args, **kw).as_subclass(Device)
            used = []
            t.record_stream = lambda s: used.append(s.cuda_stream)
            made.append((current[-1], used))
            return t
        return make

    def stream(raw, *_, **__):
        return types.SimpleNamespace(cuda_stream=raw)

    monkeypatch.setattr(sn, "_lib", library)
    monkeypatch.setattr(sn, "_raw_stream", lambda _: current[-1])
    monkeypatch.setattr(torch, "empty", recorded(torch.empty))
    monkeypatch.setattr(torch, "empty_like", recorded(torch.empty_like))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: stream(current[-1]))
    monkeypatch.setattr(torch.cuda, "stream", Entered)
    monkeypatch.setattr(torch.cuda, "ExternalStream", stream)
    for f in (sn.sn_embed_bwd_workspace, sn.sn_rmsnorm_bwd_workspace):
        f.cache_clear()                                  # (sizes that the stand-in gives are not kept)
    yield sn, library.streams, made
    for f in (sn.sn_embed_bwd_workspace, sn.sn_rmsnorm_bwd_workspace):
        f.cache_clear()


@pytest.mark.parametrize("name", NAMES)
def test_memory_is_the_given_streams(stand_in, name):
    sn, streams, made = stand_in
    call = calls(sn)[name]
    for given in (GIVEN, types.SimpleNamespace(cuda_stream=GIVEN)):
        del streams[:], made[:]
        call(given)
        assert set(streams) == {GIVEN} and made
        # allocated as the given stream's; not given again while the current one may use it
        assert all(m == (GIVEN, [CURRENT]) for m in made), made
    for given in (None, CURRENT):
        del streams[:], made[:]
        call(given)
        assert set(streams) == {CURRENT} and made and all(m == (CURRENT, []) for m in made)


def test_every_call_that_allocates_is_listed(stand_in):
    assert sorted(calls(stand_in[0])) == sorted(NAMES)


BUSY = 400_000_000                                       # cycles: some 200 ms, far longer than the calls


def overwrite(n=64 << 20):
    """Allocations of every size class on the current stream, filled with bytes that are no
    permissible value of anything: what a call left to that stream's allocator is written over."""
    kept = []
    for size in (512, 4096, 1 << 16, 1 << 18, 1 << 20, 3 << 20, 10 << 20, 20 << 20):
        for _ in range(max(1, min(64, n // size // 8))):
            kept.append(torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF))
    return kept


@pytest.mark.gpu
@pytest.mark.parametrize("raw", [False, True])
def test_calls_on_a_busy_stream(sn, raw):
    """Gradients, scores and clipping on a stream that is kept busy, with their own workspaces and
    outputs, while the current stream allocates and writes: the same bits as on the current stream."""
    T, d, V = 5000, 1024, 3000
    g = torch.Generator(device="cuda").manual_seed(5)
    x, h = (torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(d, generator=g, device="cuda")
    ids = torch.randint(V, (T,), generator=g, device="cuda", dtype=I32)
    grads = [torch.randn(n, generator=g, device="cuda") for n in (7, 3000000)]
    clipped = [torch.empty_like(t) for t in grads]
    L = sn.GradList(grads, out=clipped)
    basis = sn.Basis(torch.linalg.qr(torch.randn(d, 16, generator=g, device="cuda"))[0].contiguous())
    target = (ids % d).int()

    def run(stream):
        Y, H = sn.sn_rmsnorm_fwd(x, w, 1e-5, R=h, stream=stream)
        codes, scale, _ = sn.sn_rmsnorm_fwd_quant(x, w, 1e-5, "e4m3", group=32, stream=stream)
        dX, dw = sn.sn_rmsnorm_bwd(x, h, w, 1e-5, dH=x, stream=stream)
        dE = sn.sn_embed_bwd(x, ids, V, stream=stream)
        few = sn.sn_embed_bwd(x[:100], ids[:100], V, stream=stream)
        X = sn.sn_embed_fwd(dE, ids, stream=stream)
        logp, lse, ent, alt, alt_logp = sn.sn_logprob_fwd(x, target, top=5, stream=stream)
        norm = sn.sn_grads_clip(L, sn.sn_grads_sumsq(L, stream=stream), 1.0, stream=stream)
        TS = sn.sn_build_ts(basis, x, stream=stream)
        W = sn.sn_project_weight(basis, x[:d], stream=stream)
        return [Y, H, codes, scale, dX, dw, dE, few, X, logp, lse, ent, alt, alt_logp, norm, TS, W]

    want = run(None) + [c.clone() for c in clipped]
    overwrite()
    for turn in range(3):
        for c in clipped:
            c.zero_()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            torch.cuda._sleep(BUSY)
        got = run(side.cuda_stream if raw else side)
        kept = overwrite()
        assert not side.query()                          # the calls were still waiting
        torch.cuda.current_stream().wait_stream(side)
        got += [c.clone() for c in clipped]
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (turn, i)
        del kept, got
    basis.destroy()


@pytest.mark.gpu
def test_outputs_outlive_their_use_on_the_current_stream(sn):
    """An output that is dropped while the current stream still reads it is not given to the next
    call on the other stream."""
    T, d = 4096, 1024
    table = torch.arange(2 * d, device="cuda", dtype=F32).view(2, d)
    zeros, ones = (torch.full((T,), i, device="cuda", dtype=I32) for i in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        out = sn.sn_embed_fwd(table, zeros, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda._sleep(BUSY)
        seen = out.clone()
        del out
        sn.sn_embed_fwd(table, ones, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(seen, table[0].expand(T, d))


@pytest.mark.gpu
def test_step_on_another_stream_is_compared_whole(sn):
    """Norm, gradients and clipping given a stream, the clipped gradients read in its order."""
    T, d = 3000, 256
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(d, device="cuda")
    ids = torch.randint(700, (T,), generator=g, device="cuda", dtype=I32)
    L = sn.GradList([torch.randn(3000000, generator=g, device="cuda")])
    L2 = sn.GradList(L.grads, out=[torch.empty_like(t) for t in L.grads])
    torch.cuda.synchronize()

    def calls(stream):
        _, H = sn.sn_rmsnorm_fwd(x, w, 1e-5, R=r, stream=stream)
        dX, dw = sn.sn_rmsnorm_bwd(x, H, w, 1e-5, dH=r, stream=stream)
        dE = sn.sn_embed_bwd(dX, ids, 700, stream=stream)
        norm = sn.sn_grads_clip(L2, sn.sn_grads_sumsq(L2, stream=stream), 1.0, stream=stream)
        torch.cuda.current_stream().wait_stream(stream)
        return [H, dX, dw, dE, norm, L2.out[0].clone()]

    want = calls(torch.cuda.current_stream())
    torch.cuda.synchronize()
    L2.out[0].zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for a, b in zip(calls(side), want):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_on_a_forked_stream_of_a_capture(sn):
    """Calls on a second stream of a captured graph make their memory in the graph's pool: replays
    give the eager calls' bits."""
    T, d, V = 3000, 512, 900
    g = torch.Generator(device="cuda").manual_seed(7)
    x, h = (torch.randn(T, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(d, generator=g, device="cuda")
    ids = torch.randint(V, (T,), generator=g, device="cuda", dtype=I32)
    side = torch.cuda.Stream()

    def run():
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        dX, dw = sn.sn_rmsnorm_bwd(x, h, w, 1e-5, stream=side)
        dE = sn.sn_embed_bwd(dX, ids, V, stream=side)
        Y = sn.sn_rmsnorm_fwd(h, w, 1e-5)[0]             # meanwhile
        here.wait_stream(side)
        return [dX, dw, dE, Y]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in (1, 2):
        x.copy_(torch.randn(T, d, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = run()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), i
