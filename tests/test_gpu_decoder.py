"""The causal operators together: a decoder's serving agrees with its whole-sequence form, and it learns."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def model(**kw):
    from paper_2507_08637_amd.decoder import Decoder
    torch.manual_seed(3)
    return Decoder(**kw)


@pytest.mark.parametrize("dtype,hidden,heads", [(torch.float32, 128, 4), (torch.bfloat16, 256, 4), (torch.bfloat16, 256, 2)])
def test_prompts_and_tokens_agree_with_the_whole_sequence(dtype, hidden, heads):
    """float32: the same products in other orders, a few hundred roundings of 2^-24 through two layers.  bfloat16: activations are rounded at the same places, to 2^-9 in the
    root mean square each, about ten times a layer: sqrt(20) 2^-9 of the logits' size between two forms that round differently, twice that as the bound."""
    m = model(hidden=hidden, heads=heads, dtype=dtype)
    lengths, more = [33, 1, 90, 64], 5
    g = torch.Generator(device="cuda").manual_seed(0)
    rows = [torch.randint(64, (n + more,), generator=g, device="cuda") for n in lengths]
    whole = [m(row[None])[0].detach() for row in rows]
    weights, cache = m.serving(), m.cache(7)
    slots = torch.tensor([4, 0, 6, 2], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 33, 34, 124, 188], dtype=torch.int32, device="cuda")
    logits = m.prefill(torch.cat([r[:n] for r, n in zip(rows, lengths)]), offsets, cache, slots, weights)
    tol = 2e-5 if dtype == torch.float32 else 2 * 20 ** 0.5 * 2.0 ** -9
    def close(got, want):
        assert float((got - want).norm()) <= tol * float(want.norm()), float((got - want).norm() / want.norm())
    for b, n in enumerate(lengths):
        close(logits[int(offsets[b]):int(offsets[b + 1])], whole[b][:n])
    for t in range(more):
        tokens = torch.stack([row[n + t] for row, n in zip(rows, lengths)])
        logits = m.step(tokens, cache, slots, weights)
        close(logits, torch.stack([w[n + t] for w, n in zip(whole, lengths)]))


def test_it_learns_and_goes_on():
    """Two tokens that take turns, another two in every sequence: ln 64 = 4.2 to guess, 0.07 where only the first two tokens of 128 are guessed, 0.7 where the two are known and not whose turn it is."""
    from paper_2507_08637_amd import decoder
    m = model()
    losses = decoder.train(m, 200)
    assert losses[0] > 3.5 and sum(losses[-20:]) / 20 < 0.8
    g = torch.Generator(device="cuda").manual_seed(5)
    rows = decoder.batch(6, 64, 64, 2, g)
    prompts = [row[:n] for row, n in zip(rows, (24, 33, 40, 17, 48, 31))]
    want = torch.stack([row[len(p):len(p) + 8] for row, p in zip(rows, prompts)])
    for eight_bit in (False, True):
        got = decoder.generate(m, prompts, 8, eight_bit)
        assert float((got == want).float().mean()) > 0.8
