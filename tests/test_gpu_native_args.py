"""Arguments of the calls that the native extension marshals: what has no truth value raises its own error."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mala():
    from paper_2609_32712_b200 import mala as m
    m.lib()
    return m


def test_flags_without_a_truth_value(mala):
    both = torch.tensor([True, False])
    z = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    rot = mala.Rotary(torch.ones(8, dtype=torch.float64))
    norm = mala.HeadNorm(torch.ones(16, device="cuda"), None)
    q, pages, scales = z(1, 4, 2, 16), torch.zeros((2, 16, 1, 16), dtype=torch.uint8, device="cuda"), torch.ones((2, 1, 1), device="cuda")
    calls = [lambda flag: mala.fwd_paged_fp8(q, pages, pages, scales, scales, i32(0, 4), i32(0).view(1, 1), i32(8), 4, 8, 0.25, 0.0, causal=flag),
             lambda flag: mala.rotary_bwd(q, None, rot, norm=norm, q=q, weights=flag)]
    for call in calls:
        call(True)
        with pytest.raises(RuntimeError, match="ambiguous"):
            call(both)
    rot.interleaved = both
    with pytest.raises(RuntimeError, match="ambiguous"):
        mala.rotary(q, None, rot)
    torch.cuda.synchronize()
    assert mala.device_status() == 0


def test_packed_calls_without_offsets(mala):
    """No offsets, or those of one side only, are not the call for sequences of one length."""
    q = torch.zeros((1, 4, 2, 16), dtype=torch.bfloat16, device="cuda")
    rot, cu = mala.Rotary(torch.ones(8, dtype=torch.float64)), torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    from paper_2609_32712_b200 import autograd as A
    for a, b in ((None, None), (cu, None), (None, cu)):
        for call in (lambda: mala.rotary_varlen(q, q, a, b, rot), lambda: mala.rotary_varlen_bwd(q, q, a, b, rot), lambda: A.rotary_packed(q, q, a, b, rot)):  # noqa: B023
            with pytest.raises(AssertionError):
                call()
    assert torch.equal(mala.rotary_varlen(q, q, cu, cu, rot)[0], q)
