"""Parameters, their copies and given outputs that the library writes over: autograd knows of it, as of torch's own in-place
operations, so a backward pass that needs the old values says so.  Needs an MI355X."""
import pytest
import torch

from paper_2104_02621_amd import capscaps as cc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_parameters_and_copies_of_a_step(bits):
    w = torch.ones(300, device="cuda", requires_grad=True)
    low = torch.ones(300, device="cuda", dtype=torch.bfloat16)
    opt = cc.AdamW([w], state_bits=bits, copies=[low])
    versions = w._version, low._version
    loss = (w * w).sum()
    opt.step([torch.ones(300, device="cuda")])
    assert w._version > versions[0] and low._version > versions[1]
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    # ... also of tensors that take others' places
    opt.copies[0] = other = torch.ones(300, device="cuda", dtype=torch.float16)
    before = other._version
    opt.step([torch.ones(300, device="cuda")])
    assert other._version > before


def test_the_stream_written_over_and_given_outputs():
    x = torch.randn((5, 64), device="cuda")
    b, scale = torch.randn((5, 64), device="cuda"), torch.ones(1, device="cuda", requires_grad=True)
    h = torch.empty((5, 64), device="cuda")
    loss = (x * scale).sum()
    versions = x._version, h._version, b._version
    r = cc.block_norm_fwd(x, b, y=x, h=h)
    assert r.y is x and r.h is h
    assert x._version > versions[0] and h._version > versions[1] and b._version == versions[2]
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
