"""Outputs and scratch of the calls that run a quantized network belong to the context's stream, whichever stream is the current one."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture
def allocations(monkeypatch):
    """The handle of the stream that is current at every allocation of the binding, and how often there was one."""
    import paper_2509_05576_amd as fobq
    seen, empty = [], torch.empty

    def spy(*a, **kw):
        seen.append(torch.cuda.current_stream(0).cuda_stream)
        return empty(*a, **kw)

    class Torch:
        def __getattr__(self, name):
            return spy if name == "empty" else getattr(torch, name)

    monkeypatch.setattr(fobq.binding, "torch", Torch())
    return seen


@pytest.mark.parametrize("context_on_side", [False, True])
def test_memory_is_the_context_streams(allocations, context_on_side):
    import paper_2509_05576_amd as fobq
    default, side = torch.cuda.default_stream(0), torch.cuda.Stream(0)
    home, away = (side, default) if context_on_side else (default, side)
    with torch.cuda.stream(home):
        ctx = fobq.Ctx(0)
        x = torch.ones((4, 8192), device="cuda")
        cache = fobq.Kv4Cache(*(torch.zeros(s, dtype=t, device="cuda") for s, t in (((64, 1, 64, 64), torch.uint8),) * 2 + (((64, 1, 64), torch.int32),) * 2))
        batch = fobq.Kv4Batch(torch.arange(64, dtype=torch.int32, device="cuda")[None], torch.full((1,), 4000, dtype=torch.int32, device="cuda"))
        q = torch.ones((1, 2, 128), dtype=torch.bfloat16, device="cuda")
        many = torch.ones((64, 8192), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(away):
        calls = [lambda: ctx.fp8_quantize(x), lambda: ctx.kv4_read(cache, batch, 1), lambda: ctx.kv4_attention(cache, batch, q)]
        m = ctx.fp8_quantize(many)
        calls.append(lambda: ctx.fp8_matmul(m, m))
        for call, count in zip(calls, (2, 2, 2, 2)):             # (attention and the product: a result and scratch)
            del allocations[:]
            call()
            assert allocations == [home.cuda_stream] * count
            assert torch.cuda.current_stream(0).cuda_stream == away.cuda_stream
    torch.cuda.synchronize()
    ctx.close()
