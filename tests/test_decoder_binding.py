"""What the torch binding of a decoder's steps in 8 bits refuses beyond what the entry points do (CPU only)."""
import pytest
import torch

import paper_2404_02445_amd as P


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_an_activation_without_a_gate_is_refused(act):
    x, q = torch.zeros(3, 40), P.alloc_rows8(3, 40, "cpu")
    with pytest.raises(ValueError, match="gate"):
        P.mopar_quantize_rows(x, q, act=act)
    for kw in (dict(), dict(act=None), dict(act="none")):                    # plain rows: as far as the CPU lets them
        with pytest.raises(ValueError, match="GPU"):
            P.mopar_quantize_rows(x, q, **kw)
    for kw in (dict(gate=x), dict(gate=x, act=act)):
        with pytest.raises(ValueError, match="GPU"):
            P.mopar_quantize_rows(x, q, **kw)


def test_alternatives_of_another_shape_are_refused():
    x, tokens, lp = torch.zeros(3, 40), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    ids = torch.zeros(3, 2, dtype=torch.int32)
    for other in (torch.zeros(2, 3), torch.zeros(6), torch.zeros(3, 3), torch.zeros(2, 3).t()):
        with pytest.raises(ValueError, match="top_logprob"):
            P.mopar_token_logprobs(x, tokens, lp, top_logprob=other, top_id=ids)
    with pytest.raises(ValueError, match="GPU"):
        P.mopar_token_logprobs(x, tokens, lp, top_logprob=torch.zeros(3, 2), top_id=ids)
