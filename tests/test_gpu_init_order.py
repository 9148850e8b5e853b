"""GPU: a context that is made while the default stream is busy is ready on every other stream when dion_init returns."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

from paper_2504_05295_b200 import binding  # noqa: E402


def test_a_context_is_ready_on_every_stream():
    with binding.Dion():      # (whatever is loaded once)
        pass
    side = torch.cuda.Stream()
    good, bad = torch.ones(1000, device="cuda"), torch.full((1000,), float("nan"), device="cuda")
    long = torch.ones(5000000, device="cuda")
    out, total = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    torch.cuda._sleep(500_000_000)      # a quarter of a second
    done.record()
    with binding.Dion() as opt:
        opt.grad_norm(binding.grad_list([good]), norm_out=out, stream=side)
        opt.grad_norm(binding.grad_list([long]), norm_out=total, stream=side)
        assert opt.get_status(stream=side) == (0, 0)
        opt.grad_norm(binding.grad_list([bad]), norm_out=out, stream=side)
        side.synchronize()
        busy = not done.query()
        torch.cuda.synchronize()
        # what the call left is still there when the default stream has come to its end
        assert opt.get_status(stream=side) == (binding.STATUS_NONFINITE, 0)
    assert abs(float(total) - 5000000 ** 0.5) <= 5 * 2.0 ** -24 * 5000000 ** 0.5
    print("the default stream was", "busy" if busy else "idle", "meanwhile")
