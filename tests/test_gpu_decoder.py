"""GPU: the example layer that uses the 4-bit cache's calls together with the products of signs."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def plan(bnn, sequences, longest, kv_heads, head_dim, page=16):
    pages = -(-longest // page)
    table = torch.randperm(sequences * pages, device="cuda").to(torch.int32).view(sequences, pages)
    return table, bnn.Cache4(sequences * pages, kv_heads=kv_heads, head_dim=head_dim, page=page)


@pytest.fixture(scope="module")
def layer():
    from paper_2006_16578_amd import decoder
    return decoder.DecoderLayer(256, 8, 2, 64, 512, seed=3)


def test_a_prompt_at_once_in_chunks_and_token_by_token(layer):
    import paper_2006_16578_amd as bnn
    torch.manual_seed(0)
    x = torch.randn(3, 70, 256, device="cuda")

    def run(sizes, keep=None):
        table, cache = plan(bnn, 3, 70, 2, 64)
        lens, out, at = torch.zeros(3, dtype=torch.int32, device="cuda"), [], 0
        for n in sizes:
            lens += n
            o = layer.attention(x[:, at:at + n].reshape(-1, 256), cache, table, lens, keep=keep)
            out.append(o.view(3, n, 8, 64))
            at += n
        return torch.cat(out, 1)

    whole = run([70])
    assert torch.isfinite(whole).all() and whole.dtype == torch.float32
    # the same sums in other orders: fp32 throughout, over at most 70 keys of values around 1
    for other in (run([33, 1, 36]), run([1] * 70), run([64, 6], keep=5), run([70], keep=5)):        # five pages are all there are
        assert (other - whole).abs().max() < 1e-4
    # three pages of up to five: no more than the early tokens agree
    some = run([70], keep=3)
    assert (some[:, :48] - whole[:, :48]).abs().max() < 1e-4 and (some[:, 48:] - whole[:, 48:]).abs().max() > 1e-2


def test_forward_and_the_command(layer, capsys):
    import paper_2006_16578_amd as bnn
    from paper_2006_16578_amd import decoder
    table, cache = plan(bnn, 2, 40, 2, 64)
    lens = torch.tensor([30, 7], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 30, 37], dtype=torch.int32, device="cuda")
    y = layer.forward(torch.randn(37, 256, device="cuda"), cache, table, lens, start)
    assert y.shape == (37, 256) and torch.isfinite(y).all()
    lens += 1
    assert torch.isfinite(layer.forward(y[[29, 36]].contiguous(), cache, table, lens, keep=2)).all()
    decoder.main(["--batch", "2", "--context", "1500", "--steps", "2", "--keep", "4"])
    out = capsys.readouterr().out
    assert "attention to the whole cache" in out and "4 pages of 64 tokens" in out
