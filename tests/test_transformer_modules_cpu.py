"""Modules over the transformer operators (arxiv 2411.01238, Sections 2.1 and 4.2): what they hold, without a GPU."""
import torch

from paper_2411_01238_amd import transformer as tr


def test_modules_have_seeds_of_their_own():
    make = lambda: [tr.ElementDropout(0.5), tr.ElementDropout(0.5), tr.DropoutAddNorm(8, device="cpu"), tr.DropoutAddNorm(8, device="cpu")]     # noqa: E731
    torch.manual_seed(5)
    a = [m.seed for m in make()]
    assert len(set(a)) == 4 and all(0 <= s < 1 << 62 for s in a)
    torch.manual_seed(5)
    assert [m.seed for m in make()] == a                # a program's runs repeat
    torch.manual_seed(6)
    assert not set(a) & {m.seed for m in make()}        # ranks need not


def test_seeds_that_are_given_are_taken():
    state = torch.get_rng_state()
    assert tr.ElementDropout(0.5, seed=3).seed == 3 and tr.DropoutAddNorm(8, seed=0, device="cpu").seed == 0 and tr.ElementDropout(0.5, 7).seed == 7
    assert torch.equal(torch.get_rng_state(), state)
