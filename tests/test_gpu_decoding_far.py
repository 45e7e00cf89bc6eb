"""GPU: rows, pages and weights that lie more than 2^31 elements and 2^32 bytes into their tensors, against the same calls on small ones (which other tests hold against the oracle)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bnn():
    import paper_2006_16578_amd as b
    b.load()
    return b


@pytest.mark.parametrize("dtype,more", [(torch.bfloat16, 8), (torch.float32, 4), (torch.bfloat16, 3)])
def test_logits_far_apart(bnn, dtype, more):
    gen = torch.Generator("cuda").manual_seed(1)
    wide = torch.empty(4, (1 << 30) + more, dtype=dtype, device="cuda")
    x = wide[:, :1000].copy_(torch.randn(4, 1000, device="cuda", generator=gen))
    near = torch.empty(4, 1000 + more, dtype=dtype, device="cuda")[:, :1000].copy_(x)        # rows begin at the same places within 16 bytes
    targets = torch.tensor([0, 999, 17, 500], device="cuda")
    for a, b in zip(bnn.token_logprobs(x, targets, top=5), bnn.token_logprobs(near, targets, top=5)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_far_apart(bnn, interleaved):
    gen = torch.Generator("cuda").manual_seed(2)
    wide = torch.empty(4, 1 << 30, dtype=torch.bfloat16, device="cuda").view(4, 1 << 23, 128)
    x = wide[:, ::(1 << 23) - 1, :96].copy_(torch.randn(4, 2, 96, device="cuda", generator=gen))
    near, positions, f = x.contiguous(), torch.tensor([3, 0, 2147483647, -9], dtype=torch.int32, device="cuda"), bnn.rotary_frequencies(64)
    want = bnn.rotary(near, positions, f, interleaved=interleaved)
    assert torch.equal(bnn.rotary(x, positions, f, interleaved=interleaved), want)
    assert bnn.rotary(x, positions, f, interleaved=interleaved, out=x) is x and torch.equal(x, want)


def test_pages_far_into_the_cache(bnn):
    rng, gen = np.random.default_rng(3), torch.Generator("cuda").manual_seed(3)
    far, small = bnn.Cache4(70000, kv_heads=1, head_dim=256, page=256), bnn.Cache4(12, kv_heads=1, head_dim=256, page=256)
    assert far.data.numel() > 1 << 32
    pages = np.concatenate([[0, 69999], rng.choice(np.arange(60000, 69999), 10, replace=False)]).astype(np.int32)
    ints = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()
    lens, start, f = ints([700, 513]), ints([0, 700, 1213]), bnn.rotary_frequencies(256)
    q, k, v = (torch.randn(1213, h, 256, device="cuda", generator=gen).bfloat16() for h in (2, 1, 1))
    results = []
    for cache, page in ((far, pages), (small, np.arange(12))):
        table, into = ints([page[:3], page[3:6]]), ints([page[6:8], page[8:10]])
        turned = cache.write_rotary(q, k, v, table, lens, f, start)
        out, lse = cache.attend(turned, table, lens, start, want_lse=True)
        w = cache.weigh(turned, lse, table, lens, start, out=torch.zeros(2, 1, 768, device="cuda"))
        one = cache.weigh(turned[:2].contiguous(), lse[:2].contiguous(), table, lens, previous=w)
        tokens, kept = cache.heaviest(w, table, lens, 400, 4, 50)
        moved = cache.move(tokens, table, into, w)
        results.append((turned, out, w, one[:, :, :513], tokens, kept, moved, *cache.read(into, kept, ints([0, 400, 800]), tokens=800)))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert (results[0][2] > 0).sum() == 1213


def test_weights_far_apart(bnn):
    gen = torch.Generator("cuda").manual_seed(4)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    cache = bnn.Cache4(8, kv_heads=3, head_dim=64, page=16)
    table, into, lens = ints([[0, 1, 2]]), ints([[4, 5]]), ints([41])
    q, k, v = (torch.randn(41, 3, 64, device="cuda", generator=gen) for _ in range(3))
    cache.write(k, v, table, lens)
    _, lse = cache.attend(q, table, lens, want_lse=True)
    results = []
    for width in (48, (1 << 30) + 1):
        w = torch.empty(1, 3, width, device="cuda")
        w[:, :, :41] = 0.5
        cache.weigh(q, lse, table, lens, out=w)
        cache.weigh(q[:5].contiguous(), lse[:5].contiguous(), table, lens, previous=w, decay=0.5, out=w)
        tokens, kept = cache.heaviest(w, table, lens, 20, 1, 3)
        results.append((w[:, :, :41].clone(), tokens, kept, cache.move(tokens, table, into, w)))
        del w
    for a, b in zip(*results):
        assert torch.equal(a, b)
