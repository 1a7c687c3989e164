"""examples/kv4_samples.py: samples that share their prompt's pages are what samples with pages of their own are, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from examples import kv4_samples
    return kv4_samples


@pytest.mark.parametrize("prompt,samples,steps", [(150, 3, 40), (64, 2, 70), (1, 4, 5)])
def test_shared_pages_give_what_pages_of_ones_own_give(example, prompt, samples, steps):
    import torch
    g = torch.Generator(device="cuda").manual_seed(prompt)
    tokens = torch.randint(0, 1000, (prompt,), device="cuda", generator=g)
    noise = 3 * torch.randn(steps, samples, 1000, device="cuda", generator=g)
    one, logits, rows = example.generate(example.Decoder(), tokens, noise)
    two, own, apart = example.generate(example.Decoder(), tokens, noise, share=False, compact_every=7)
    assert torch.equal(one, two) and torch.equal(logits.view(torch.int16), own.view(torch.int16))
    assert torch.isfinite(logits).all() and len(set(map(tuple, one.T.tolist()))) == samples
    whole = (prompt // 64) * (samples - 1)                        # pages that are held once instead of by every sample
    assert int((apart.refs > 0).sum()) - int((rows.refs > 0).sum()) == whole
    for r in (rows, apart):
        held = torch.bincount(r.table[r.table >= 0].long(), minlength=len(r.refs))
        assert torch.equal(held.int(), r.refs)


def test_a_sample_that_ends_gives_its_place_to_another(example):
    """Behind the step the two rows go on from the same history: with the same noise they stay the same."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(9)
    tokens = torch.randint(0, 1000, (70,), device="cuda", generator=g)
    noise = 3 * torch.randn(30, 3, 1000, device="cuda", generator=g)
    noise[11:, 0] = noise[11:, 2]
    out, logits, rows = example.generate(example.Decoder(), tokens, noise, drop_at=10)
    assert torch.equal(out[11:, 0], out[11:, 2]) and not torch.equal(out[:11, 0], out[:11, 2])
    assert torch.equal(logits[0].view(torch.int16), logits[2].view(torch.int16))
    held = torch.bincount(rows.table[rows.table >= 0].long(), minlength=len(rows.refs))
    assert torch.equal(held.int(), rows.refs)
