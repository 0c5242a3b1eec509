"""Sizes past 32 bits do not reach the C calls, whose 32-bit arguments would take what is left of them."""
import pytest
import torch

import paper_2210_15748_amd as dz

META = torch.device("meta")


def meta_index():
    """A handle-less index for tensors without memory: the binding's own checks raise before the library sees the call."""
    return dz.Index(None, dz.Config(d=128, L=32, C=7), META)


def outputs(n, top):
    return (torch.empty(n, device=META), torch.empty(n, device=META), torch.empty(n, top, dtype=torch.uint32, device=META),
            torch.empty(n, top, device=META))


def test_a_vocabulary_past_32_bits_is_refused():
    V = (1 << 32) + 5
    a, b = torch.empty(3, 4, dtype=torch.int8, device=META), torch.empty(V, 4, dtype=torch.int8, device=META)
    with pytest.raises(ValueError, match="vocab has 4294967301 rows"):
        dz.head_logprobs(meta_index(), a, torch.empty(3, device=META), b, torch.empty(V, device=META), None, 2, outs=outputs(3, 2),
                         workspace=torch.empty(256, dtype=torch.uint8, device=META))


@pytest.mark.parametrize("top", [1 << 32, (1 << 32) + 3, -1])
def test_a_number_of_alternatives_past_32_bits_is_refused(top):
    x = torch.empty(1, 100, device=META)
    with pytest.raises(ValueError, match="n_top"):
        dz.token_logprobs(meta_index(), x, None, top, workspace=torch.empty(256, dtype=torch.uint8, device=META))
    with pytest.raises(ValueError, match="n_top"):
        dz.head_logprobs(meta_index(), x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0], None, top,
                         workspace=torch.empty(256, dtype=torch.uint8, device=META))


@pytest.mark.parametrize("rows", [1, 2])
def test_columns_past_32_bits_are_refused(rows):
    k = (1 << 32) + 8
    a = torch.empty(rows, k, dtype=torch.int8, device=META)
    x, s = torch.empty(rows, k, dtype=torch.float16, device=META), torch.empty(rows, device=META)
    ws = torch.empty(256, dtype=torch.uint8, device=META)
    with pytest.raises(ValueError, match="a has . rows of 4294967304"):
        dz.scaled_matmul(meta_index(), a, s, a, s, out=torch.empty(rows, rows, device=META), workspace=ws)
    with pytest.raises(ValueError, match="logits has . rows of 4294967304"):
        dz.token_logprobs(meta_index(), x, None, 2, outs=outputs(rows, 2), workspace=ws)
    with pytest.raises(ValueError, match="x has . rows of 4294967304"):
        dz.quantize_rows(meta_index(), x, out=a, out_scales=s)
