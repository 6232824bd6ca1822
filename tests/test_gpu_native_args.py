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
