"""GPU: the example layer with rotary positions, weights of cached tokens and eviction, and the head's log probabilities."""
import numpy as np
import pytest
import torch

from oracle import decoding as od

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layer():
    from paper_2006_16578_amd import decoder
    return decoder.DecoderLayer(256, 8, 2, 64, 512, seed=3, rotary_base=10000.0)


def plan(sequences, longest, page=16, spare=0):
    import paper_2006_16578_amd as bnn
    pages = -(-longest // page)
    order = torch.randperm(sequences * (pages + spare), device="cuda").to(torch.int32)
    return order[:sequences * pages].view(sequences, pages), order[sequences * pages:].view(sequences, -1), bnn.Cache4(sequences * (pages + spare), kv_heads=2, head_dim=64, page=page)


def test_positions_make_the_order_count(layer):
    """At once, in chunks and token by token the same (fp32 sums in other orders, over at most 70 keys of values around 1); without positions another result."""
    from paper_2006_16578_amd import decoder
    torch.manual_seed(0)
    x = torch.randn(3, 70, 256, device="cuda")

    def run(layer, sizes):
        table, _, cache = plan(3, 70)
        lens, out, at = torch.zeros(3, dtype=torch.int32, device="cuda"), [], 0
        for n in sizes:
            lens += n
            out.append(layer.attention(x[:, at:at + n].reshape(-1, 256), cache, table, lens).view(3, n, 8, 64))
            at += n
        return torch.cat(out, 1)
    whole = run(layer, [70])
    assert torch.isfinite(whole).all()
    for other in (run(layer, [33, 1, 36]), run(layer, [1] * 70)):
        assert (other - whole).abs().max() < 1e-4
    plain = decoder.DecoderLayer(256, 8, 2, 64, 512, seed=3)
    assert torch.equal(plain.w_qkv, layer.w_qkv) and plain.frequencies is None
    assert (run(plain, [70]) - whole).abs().max() > 1e-2
    # positions that are given are taken: the same as counted, and further on the same angles between tokens
    table, _, cache = plan(3, 70)
    lens = torch.full((3,), 70, dtype=torch.int32, device="cuda")
    counted = torch.arange(70, dtype=torch.int32, device="cuda").repeat(3)
    assert torch.equal(layer.attention(x.reshape(-1, 256), cache, table, lens, positions=counted).view(3, 70, 8, 64), whole)


def test_weights_of_steps_add_up(layer):
    torch.manual_seed(1)
    x = torch.randn(2, 60, 256, device="cuda")
    sums = []
    for sizes in ([60], [25, 1, 1, 33], [1] * 60):
        table, _, cache = plan(2, 60)
        lens, at, weights = torch.zeros(2, dtype=torch.int32, device="cuda"), 0, torch.zeros(2, 2, 64, device="cuda")
        for n in sizes:
            lens += n
            layer.attention(x[:, at:at + n].reshape(-1, 256), cache, table, lens, weights=weights)
            at += n
        sums.append(weights)
        # every row of four query heads a kv head gives 1; fp32 sums of up to 60 weights of scores below 100
        assert ((weights.sum(-1) - 60 * 4).abs() <= 240 * (60 + 100 * 72) * 2.0 ** -24).all() and (weights[..., 60:] == 0).all()
    for other in sums[1:]:
        assert ((other - sums[0]).abs() <= 2 * (60 + 100 * 72) * 2.0 ** -24 * sums[0]).all()
    with pytest.raises(ValueError):
        layer.attention(x[:, :1].reshape(-1, 256), cache, table, lens, keep=3, weights=weights)


def test_generating_under_a_budget(layer):
    """Steps with eviction whenever 64 tokens are passed: the cache stays within its pages, positions go on, all finite; what is kept are the first, the last and the heaviest."""
    from paper_2006_16578_amd import decoder
    torch.manual_seed(2)
    head = decoder.Head(256, 1000, seed=4)
    table, spare, cache = plan(2, 80, spare=5)
    lens, weights = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, 80, device="cuda")
    positions = torch.zeros(2, dtype=torch.int32, device="cuda")
    x, total, cuts = torch.randn(2, 256, device="cuda"), 0.0, 0
    for step in range(150):
        lens = lens + 1
        x = layer.forward(x, cache, table, lens, positions=positions, weights=weights)
        positions += 1
        said = head.forward(x, torch.tensor([step, 999 - step], device="cuda"), top=3)
        assert torch.isfinite(said.logprobs).all() and (said.top_logprobs[:, 0] >= said.logprobs).all()
        if int(lens[0]) == 65:
            before = weights.clone()
            lens, weights = decoder.cut_back(cache, weights, table, lens, spare, 48, first=2, last=16)
            table, spare = spare, table
            kept, _ = od.heaviest(before.cpu().numpy(), spare.cpu().numpy(), np.array([65, 65]), 48, 2, 16, 16, len(cache.data))
            assert lens.tolist() == [48, 48]
            want = np.take_along_axis(before.cpu().numpy(), kept, 2)
            assert np.array_equal(weights[..., :48].cpu().numpy(), want) and (weights[..., 48:] == 0).all()
            cuts += 1
    assert cuts == 6 and torch.isfinite(x).all() and positions.tolist() == [150, 150]


def test_head(layer):
    """The head's sums are whole numbers, so its logits are exact up to one scale."""
    import paper_2006_16578_amd as bnn
    from paper_2006_16578_amd import decoder
    torch.manual_seed(3)
    head, x = decoder.Head(256, 777, seed=5), torch.randn(9, 256, device="cuda")
    targets = torch.randint(0, 777, (9,), device="cuda")
    sums = bnn.bmm(bnn.sign_pack_f32(x, 8), head.w, 256)
    for temperature in (1.0, 0.5):
        said = head.forward(x, targets, top=5, temperature=temperature)
        logits = sums.double() * (256 ** -0.5 / temperature)
        want = torch.log_softmax(logits, 1)
        # logits of up to 256 / 16 * 2; fp32 roundings of them and of sums of 777 terms
        assert ((said.logprobs.double() - want.gather(1, targets[:, None])[:, 0]).abs() <= 300 * 2.0 ** -24 * 5).all()
        assert ((said.entropy.double() + (want.exp() * want).sum(1)).abs() <= 300 * 2.0 ** -24 * 8).all()
        assert ((said.top_logprobs.double() - want.topk(5).values).abs() <= 300 * 2.0 ** -24 * 5).all()
        assert torch.equal(sums.gather(1, said.top_tokens.long()), sums.topk(5).values)
    assert head.forward(x).logprobs is None


def test_the_command(capsys):
    from paper_2006_16578_amd import decoder
    decoder.main(["--batch", "2", "--context", "1500", "--steps", "2", "--keep", "4", "--budget", "700"])
    out = capsys.readouterr().out
    assert "2 sequences of 703 tokens, attention to what is left of 1500" in out and "the likeliest next tokens" in out
