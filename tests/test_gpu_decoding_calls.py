"""GPU: the native module's forms of the calls around the cache and behind the head against binding.py's own, and calls out of the ordinary."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bnn():
    import paper_2006_16578_amd as b
    b.load()
    return b


def tensors_of(r):
    return [r] if torch.is_tensor(r) else [t for t in r if t is not None]


class Case:
    """A call: f(*tensors) with everything else fixed; written: the cache, which is looked at too."""

    def __init__(self, name, f, tensors, cache=None):
        self.name, self.f, self.tensors, self.cache = name, f, tensors, cache

    def __call__(self, *tensors):
        r = self.f(*(tensors or self.tensors))
        return tensors_of(r) + ([self.cache.data.clone()] if self.cache is not None else [])


def cases(bnn):
    g = torch.Generator(device="cuda").manual_seed(7)
    real = lambda *s: torch.randn(*s, device="cuda", generator=g)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    cache = bnn.Cache4(kv_heads=2, head_dim=64, page=16, data=torch.zeros(12, 2, bnn.load().bnn_cache4_record_bytes(64, 16, 1), dtype=torch.uint8, device="cuda"))
    table, lens, start, into = ints([[0, 1, 2], [3, 4, 5]]), ints([40, 33]), ints([0, 3, 5]), ints([[6, 7], [8, 9]])
    k, v, q = real(5, 2, 64), real(5, 2, 64), real(5, 6, 64)
    f, p = bnn.rotary_frequencies(32), ints([5, 6, 7, 8, 1000000])
    cache.write(real(73, 2, 64), real(73, 2, 64), table, lens, start=ints([0, 40, 73]))
    lse, weights = real(5, 6), real(2, 2, 50).abs()
    tokens, _ = cache.heaviest(weights, table, lens, 9, 1, 2)
    logits, targets = real(3, 900), torch.randint(0, 900, (3,), device="cuda", generator=g)
    zero = lambda: torch.zeros(2, 2, 50, device="cuda")
    return [Case("rotary", lambda q, p, f: bnn.rotary(q, p, f, interleaved=True, magnitude=1.5, inverse=True), (q, p, f)),
            Case("rotary", lambda q, p, f: bnn.rotary(q, p, f), (q.to(torch.bfloat16), p, f)),
            Case("cache4_write_rotary", lambda q, k, v, table, lens, f, start, p: cache.write_rotary(q, k, v, table, lens, f, start=start, positions=p, magnitude=1.25),
                 (q, k, v, table, lens, f, start, p), cache),
            Case("cache4_write_rotary", lambda q, k, v, table, lens, f: cache.write_rotary(q, k, v, table, lens, f, interleaved=True), (q[:4].half(), k[:4].half(), v[:4].half(), table, lens, f), cache),
            Case("cache4_weigh", lambda q, lse, table, lens, start, weights: cache.weigh(q, lse, table, lens, start=start, window=9, previous=weights, decay=0.5, out=zero()),
                 (q, lse, table, lens, start, weights)),
            Case("cache4_weigh", lambda q, lse, table, lens: cache.weigh(q, lse, table, lens, scale=0.2, causal=False)[:, :, :33], (q[:4], lse[:4], table, lens)),
            Case("cache4_heaviest", lambda weights, table, lens: cache.heaviest(weights, table, lens, 11, 2, 3), (weights, table, lens)),
            Case("cache4_move", lambda tokens, table, into, weights: cache.move(tokens, table, into, weights=weights), (tokens, table, into, weights), cache),
            Case("token_logprobs", lambda logits, targets: bnn.token_logprobs(logits, targets, scale=0.7, top=4), (logits, targets)),
            Case("token_logprobs", lambda logits, targets: bnn.token_logprobs(logits, targets), (logits[:, 3:700].to(torch.bfloat16), targets))]


class Unlistened(torch.Tensor):
    pass


def equal(a, b):
    return len(a) == len(b) and all(x.dtype == y.dtype and x.shape == y.shape and torch.equal(x, y) for x, y in zip(a, b))


def test_native_and_not(bnn, monkeypatch):
    from paper_2006_16578_amd import binding
    binding._load_native()
    native, served = binding._native, []

    class Counted:
        def __getattr__(self, name):
            f = getattr(native, name)
            return lambda *a: served.append((name, f(*a))) or served[-1][1]

    off = type("Off", (), {"__getattr__": lambda s, n: lambda *a: None})()
    for case in cases(bnn):
        monkeypatch.setattr(binding, "_native", Counted())
        fast = case()
        name, result = served.pop()
        assert name == case.name and result is not None, case.name
        monkeypatch.setattr(binding, "_native", off)
        slow = case()
        assert equal(fast, slow), case.name
        monkeypatch.setattr(binding, "_native", Counted())
        # a subclass of tensors is served by Python; another stream natively; leaves that require gradients give results that do not
        got = case(*(t.as_subclass(Unlistened) for t in case.tensors))
        assert served.pop()[1] is None and equal([t.as_subclass(torch.Tensor) for t in got], slow), case.name
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            got = case()
        stream.synchronize()
        assert served.pop()[1] is not None and equal(got, slow), case.name
        got = case(*(t.clone().requires_grad_() if t.is_floating_point() and t.dtype != torch.float64 else t for t in case.tensors))
        assert equal(got, slow) and not any(t.requires_grad for t in got), case.name
        served.clear()


def test_refused_by_type_device_and_layout(bnn):
    for case in cases(bnn):
        for i, t in enumerate(case.tensors):
            for bad in (t.cpu(), t.to(torch.complex64)):
                with pytest.raises(TypeError):
                    case(*case.tensors[:i], bad, *case.tensors[i + 1:])
            with pytest.raises((ValueError, RuntimeError)):
                case(*case.tensors[:i], t.unsqueeze(0).unsqueeze(0).unsqueeze(0), *case.tensors[i + 1:])
            if t.dim() > 1 and t.shape[-1] > 1 and t.shape[0] > 1:
                with pytest.raises(ValueError):
                    case(*case.tensors[:i], t.transpose(0, -1).contiguous().transpose(0, -1), *case.tensors[i + 1:])


def test_a_tensor_without_a_pointer_raises(bnn):
    for case in cases(bnn):
        for i in range(len(case.tensors)):
            bad = case.tensors[i].clone()
            torch._C._set_throw_on_mutable_data_ptr(bad)
            with pytest.raises(RuntimeError, match="data pointer"):
                case(*case.tensors[:i], bad, *case.tensors[i + 1:])
        case()


def test_two_streams_at_once(bnn):
    """Calls of two streams do not share memory: each has its own workspace and outputs."""
    torch.manual_seed(0)
    xs = [torch.randn(5, 70001, device="cuda") for _ in range(2)]
    ts = [torch.randint(0, 70001, (5,), device="cuda") for _ in range(2)]
    table = torch.randperm(2000, device="cuda").to(torch.int32).view(2, 1000)
    cache = bnn.Cache4(2000, kv_heads=2, head_dim=64, page=64)
    lens = torch.tensor([64000, 50000], dtype=torch.int32, device="cuda")
    ws = [torch.rand(2, 2, 64000, device="cuda") for _ in range(2)]
    want = [(bnn.token_logprobs(x, t, top=9), cache.heaviest(w, table, lens, 3000, 1, 5)) for x, t, w in zip(xs, ts, ws)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((bnn.token_logprobs(xs[i], ts[i], top=9), cache.heaviest(ws[i], table, lens, 3000, 1, 5)))
    torch.cuda.synchronize()
    for i in range(2):
        for r in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(r[0], want[i][0])) and all(torch.equal(a, b) for a, b in zip(r[1], want[i][1]))


def test_numbers_that_are_no_python_numbers(bnn):
    x, t = torch.randn(3, 50, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(bnn.token_logprobs(x, t, scale=np.float64(0.5), top=np.int64(3)), bnn.token_logprobs(x, t, scale=0.5, top=3)))
    p, f = torch.arange(3, dtype=torch.int32, device="cuda"), bnn.rotary_frequencies(16)
    y = torch.randn(3, 2, 16, device="cuda")
    assert torch.equal(bnn.rotary(y, p, f, interleaved=1, magnitude=2), bnn.rotary(y, p, f, interleaved=True, magnitude=2.0))
