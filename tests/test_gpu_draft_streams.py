"""A DraftHead made on another stream than its refiner's: its weights are ready for both."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_02438_gb300 import workloads as W  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
H, V, B, b = 512, 2080, 8, 2


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02438_gb300 import binding, build
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("made_on", ["default", "third"])
@pytest.mark.parametrize("used_on", ["refiner", "maker"])
def test_head_made_on_another_stream(X, made_on, used_on):
    from paper_2608_02438_gb300 import draft_head as D
    side = torch.cuda.Stream()
    w = W.make_weights(H, V, 256, B, W.BF16, 51, "strong")
    weights = {k: X.to_device(v, X.XPRESS_BF16) for k, v in w.items()}
    torch.cuda.synchronize()
    ref = X.Refiner(weights, H, V, 256, B, X.XPRESS_BF16, stream=side)
    g = torch.Generator(device="cuda")
    g.manual_seed(52)
    W_ready = (torch.randn((V, H), device="cuda", generator=g) * 0.1).to(BF16)
    x = torch.randn((b, B, H), device="cuda", generator=g).to(BF16)
    norm = torch.ones(H, dtype=BF16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        want = D.DraftHead(ref, norm, W_ready).base_logits(x)
    torch.cuda.synchronize()
    maker = torch.cuda.current_stream() if made_on == "default" else torch.cuda.Stream()
    with torch.cuda.stream(maker):
        torch.cuda._sleep(100_000_000)           # some 50 ms before the weights are there
        W_lm = W_ready.clone()
        head = D.DraftHead(ref, norm, W_lm)
        del W_lm                                 # its memory may be given out again on this stream
        torch.full((V, H), float("nan"), dtype=BF16, device="cuda")
    with torch.cuda.stream(side if used_on == "refiner" else maker):
        out = head.base_logits(x)                # (a refinement would not change what is tested)
    torch.cuda.synchronize()
    assert torch.equal(out["s"], want["s"]) and torch.equal(out["draft"], want["draft"])
    ref.close()
