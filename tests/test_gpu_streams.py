"""Calls on a stream that is not the current one.  What such a call allocates itself has to be that stream's memory: here the current stream is busy, and then writes to blocks of the
same sizes that are free again for whoever asks the current stream's pool next."""
import pytest
import torch

from cache_cases import make_cache, to_cache

pytestmark = pytest.mark.gpu


class BusyCurrentStream:
    """Tens of milliseconds of products on the current stream, then 0xFF written to 64 blocks of each size, which are freed."""

    def __init__(self, *sizes):
        a = torch.randn(8192, 8192, device="cuda")
        torch.cuda.synchronize()
        for _ in range(4):
            a = a @ a * 1e-2
        self.blocks = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(64)]
        self.at = {b.data_ptr() for b in self.blocks}
        del self.blocks
        for n in sizes:                                         # (this is what whoever asks the current stream's pool is given)
            assert torch.empty(n, dtype=torch.uint8, device="cuda").data_ptr() in self.at

    def check(self, side, *results):
        """The results as they are once `side` is done and as they are in the end; none of them in a block that the current stream is still to write."""
        side.synchronize()
        torch.cuda.synchronize()
        for r in results:
            assert r.data_ptr() not in self.at


def small_cache(lengths=(700, 33, 256), width=90, spare=40):
    import paper_2501_16385_amd as fbq
    return to_cache(fbq, *make_cache(list(lengths), 2, 64, 16, torch.float16, spare=spare, seed=4, width=width))


@pytest.mark.parametrize("width", [90, 44])
def test_attention_result_and_workspace(width):
    import paper_2501_16385_amd as fbq
    cache, q = small_cache(width=width), torch.randn(3, 4, 64).half().cuda()
    want, side = fbq.attention(cache, 0, q), torch.cuda.Stream()
    room = fbq.attention_workspace(cache, q).numel()
    for _ in range(3):
        busy = BusyCurrentStream(q.numel() * 2, room)
        got = fbq.attention(cache, 0, q, stream=side)
        busy.check(side, got)
        assert torch.equal(got, want)


def test_attention_result_is_kept_for_the_current_stream():
    """Freed while the current stream still has work to do with it: the side stream's next result gets other memory."""
    import paper_2501_16385_amd as fbq
    cache, q = small_cache(), torch.randn(3, 4, 64).half().cuda()
    want, side = fbq.attention(cache, 0, q), torch.cuda.Stream()
    a = torch.randn(8192, 8192, device="cuda")
    torch.cuda.synchronize()
    got = fbq.attention(cache, 0, q, stream=side)
    side.synchronize()
    for _ in range(4):
        a = a @ a * 1e-2
    copy = got.clone()
    del got
    for _ in range(8):
        fbq.attention(cache, 0, q * 3, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(copy, want)


def test_reserve():
    import paper_2501_16385_amd as fbq
    a, b, side = small_cache(), small_cache(), torch.cuda.Stream()
    count = torch.tensor([5, 40, 0], dtype=torch.int32, device="cuda")
    want = fbq.cache_reserve(a, count)
    busy = BusyCurrentStream(12)
    got = fbq.cache_reserve(b, count, stream=side)
    busy.check(side, got)
    assert torch.equal(got, want) and torch.equal(a.table, b.table) and torch.equal(a.lengths, b.lengths) and torch.equal(a.refs, b.refs)


@pytest.mark.parametrize("operation", ["fork", "compact"])
def test_workspace_of_page_operations(operation):
    import paper_2501_16385_amd as fbq

    def cache():
        c = small_cache((100, 33, 0, 0), width=10)
        c.pool.nan_to_num_(0.0)
        return c

    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    a, b, side = cache(), cache(), torch.cuda.Stream()
    parent, child = ints(0, 1), ints(2, 3)
    call = (lambda c, **kw: fbq.cache_fork(c, parent, child, **kw)) if operation == "fork" else (lambda c, **kw: fbq.cache_compact(c, **kw))
    call(a)
    room = max(t.numel() for rooms in a._rooms.values() for _, t in rooms)
    busy = BusyCurrentStream(room)
    call(b, stream=side)
    busy.check(side, *[t for rooms in b._rooms.values() for _, t in rooms])
    assert all(torch.equal(x, y) for x, y in ((a.pool, b.pool), (a.table, b.table), (a.refs, b.refs), (a.lengths, b.lengths)))
    # the same operation on the current stream goes on with memory of its own
    call(b)
    assert len(b._rooms) == 2


def layer(N=640, K=1152, r=16, seed=3):
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.random_layers import random_layer
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return random_layer(fbq.Desc(N, K, r, 4), gen, gain=0.5)


@pytest.mark.parametrize("name,M", [(n, M) for n in ("linear", "linear_unfused", "linear_static", "linear_group") for M in (1, 2, 9, 40, 72, 300)
                                    if M <= 16 or n in ("linear", "linear_group")])
def test_linears(name, M):
    import paper_2501_16385_amd as fbq
    l, x, side = layer(), torch.randn(M, 1152, device="cuda").half(), torch.cuda.Stream()
    call = (lambda **kw: fbq.linear_group([l, l], [x, x], **kw)) if name == "linear_group" else (lambda **kw: [getattr(fbq, name)(l, x, **kw)])
    want = call()
    busy = BusyCurrentStream(M * 640 * 2, max(1, fbq.workspace_bytes(l.desc, M)))
    got = call(stream=side)
    busy.check(side, *got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_quantizer_reconstruction_and_gram():
    import paper_2501_16385_amd as fbq
    l, side = layer(), torch.cuda.Stream()
    W, X = torch.randn(640, 1152, device="cuda").half() * 0.02, torch.randn(300, 1152, device="cuda").half()
    for sizes, call in (((640 * 1152 * 4,), lambda **kw: [fbq.reconstruct(l, **kw)]),
                        ((640 * 1152,), lambda **kw: [fbq.unpack_codes(l, **kw)]),
                        ((640 * 1152 // 2, 640 * 9 * 2), lambda **kw: (lambda q: [q.qweight, q.scales, q.zeros])(fbq.quantize_feedback(l.desc, W, l.At, l.Bt, **kw))),
                        ((1152 * 1152 * 2, max(256, fbq.train_workspace_bytes(l.desc, 300))), lambda **kw: [fbq.gram(l.desc, X, 1 / 300, **kw)])):
        want = call()
        busy = BusyCurrentStream(*sizes)
        got = call(stream=side)
        busy.check(side, *got)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), sizes


def test_a_step_of_the_decode_loop_keeps_what_its_layers_were_given():
    from paper_2501_16385_amd.decode_loop import DecoderStack, random_stack
    stacks = [DecoderStack(random_stack(2, 256, 640, 16, 4, seed=3), 256, 640, keep_per_layer_buffers=True, batch=2) for _ in range(2)]
    x0 = torch.randn(2, 256, device="cuda").half()
    for s in stacks:
        s.x.copy_(x0)
    stacks[0].step()
    side, busy = torch.cuda.Stream(), BusyCurrentStream(1024)
    stacks[1].step(side)
    busy.check(side)
    for a, b in zip(stacks[0].buf, stacks[1].buf):
        assert torch.equal(a["x_in"], b["x_in"]) and torch.equal(a["down"], b["down"])
    assert torch.equal(stacks[1].buf[0]["x_in"], x0) and torch.equal(stacks[0].x, stacks[1].x)
