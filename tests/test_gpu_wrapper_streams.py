"""Op-level calls on a stream of their own, beside work that is still queued on the current
one: neither may overwrite memory that the other uses."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _calls():
    """name: the call on a stream, its result known from a call without one"""
    import paper_2608_10362_gb300 as pkg
    g = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    x, w = mk(8, 512), mk(4096, 512)
    z, u = torch.randn(64, 4096, device="cuda", generator=g), torch.rand(64, device="cuda", generator=g)
    a, b, ids = mk(2, 64, 512), mk(2, 4096, 64), torch.tensor([0, 1, -1, 1, 0, 0, 1, 0], dtype=torch.int32, device="cuda")
    q = torch.randint(0, 256, (4096, 256), dtype=torch.uint8, device="cuda", generator=g)
    s, zp = mk(4096, 4).abs(), torch.full((4096, 4), 8, dtype=torch.uint8, device="cuda")
    packed = pkg.int4_pack(q, s, zp)
    return {"linear": lambda s_: pkg.op_linear(x, w, stream=s_),
            "linear_noalloc": lambda s_: pkg.op_linear_noalloc(x, w, stream=s_),
            "int4_pack": lambda s_: pkg.int4_pack(q, s, zp, stream=s_),
            "linear_int4": lambda s_: pkg.op_linear_int4(x, packed, 4096, stream=s_),
            "sample_filtered": lambda s_: pkg.op_sample_filtered(z, u, top_p=0.9, stream=s_),
            "filter_logits": lambda s_: pkg.op_filter_logits(z, top_p=0.9, stream=s_),
            "lora": lambda s_: pkg.op_lora(x, a, b, ids, stream=s_)}


@pytest.mark.parametrize("name", ["linear", "linear_noalloc", "int4_pack", "linear_int4", "sample_filtered",
                                  "filter_logits", "lora"])
def test_calls_beside_queued_work_on_the_current_stream(name):
    """Blocks of every size that the call may ask for are freed on the current stream while a
    copy from them is queued behind a long kernel there; then the call runs on another."""
    call = _calls()[name]
    want = call(None)
    side = torch.cuda.Stream()
    call(side)                                     # first use: whatever is loaded lazily
    torch.cuda.synchronize()
    sizes = [1 << k for k in range(9, 24)] + [want.nbytes]
    kept = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    freed = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)                  # some 25 ms
    for k, f in zip(kept, freed):
        k.copy_(f)
    del f, freed
    got = call(side)
    side.synchronize()
    result = got.clone()
    torch.cuda.synchronize()
    assert torch.equal(result, want)
    assert all(bool((k == 7).all()) for k in kept)
    # and the result's memory is not handed out on `side` while the current stream uses it
    torch.cuda._sleep(50_000_000)
    copy = torch.empty_like(got)
    copy.copy_(got)
    del got
    with torch.cuda.stream(side):
        for n in sizes:
            torch.full((n,), 9, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(copy, want)


@pytest.mark.parametrize("name", ["linear", "sample_filtered", "filter_logits", "lora"])
def test_temporaries_live_until_the_stream_of_the_call_is_done(name):
    """Inputs that are freed when the call returns, while the stream has not begun with it: their
    memory is not written by what the current stream does next."""
    import paper_2608_10362_gb300 as pkg
    g = torch.Generator(device="cuda").manual_seed(6)
    mk = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()
    x, w, a, b = mk(8, 512), mk(4096, 512), mk(2, 64, 512), mk(2, 4096, 64)
    ids, base = torch.tensor([0, 1, -1, 1, 0, 0, 1, 0], dtype=torch.int32, device="cuda"), mk(8, 4096).float()
    z, u, p = mk(64, 4096).float(), torch.rand(64, device="cuda", generator=g), torch.full((64,), 0.9, device="cuda")
    c = torch.Tensor.clone
    call = {"linear": lambda s: pkg.op_linear(c(x), c(w), stream=s),
            "sample_filtered": lambda s: pkg.op_sample_filtered(c(z), c(u), top_p=c(p), stream=s),
            "filter_logits": lambda s: pkg.op_filter_logits(c(z), top_p=c(p), stream=s),
            "lora": lambda s: pkg.op_lora(c(x), c(a), c(b), c(ids), base=c(base), stream=s)}[name]
    want = call(None)
    side = torch.cuda.Stream()
    call(side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)             # some 50 ms: the copies are complete long before
    got = call(side)
    for n in [1 << k for k in range(9, 23)]:
        for _ in range(4):
            torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(got, want)
