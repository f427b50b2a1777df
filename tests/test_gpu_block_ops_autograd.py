"""The decoder block's operators where autograd records: what the caller gives is used as it is where nothing
is recorded."""
import pytest

torch = pytest.importorskip("torch")
import paper_2606_27216_amd as hm

pytestmark = pytest.mark.gpu


def test_attentions_workspace_is_used_where_autograd_records():
    print("[gpu-case] attention workspace under autograd", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(1, n, h, 64, generator=gen, device="cuda") for n, h in ((1, 4), (4096, 2), (4096, 2)))
    want = hm.attention(q, k, v)
    small, room = (torch.zeros(n, dtype=torch.uint8, device="cuda") for n in (16, 1 << 26))
    with pytest.raises(hm.HimuonError):
        hm.attention(q, k, v, workspace=small)
    q.requires_grad_()
    with pytest.raises(hm.HimuonError):
        hm.attention(q, k, v, workspace=small)
    assert not room.any()
    out, lse = hm.attention(q, k, v, workspace=room)
    assert out.requires_grad and torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert room.any()  # (the keys' pieces met there)
    out.sum().backward()
    assert bool(q.grad.isfinite().all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with pytest.raises(hm.HimuonError):
        hm.attention(q, k, v, workspace=small, stream=side)
