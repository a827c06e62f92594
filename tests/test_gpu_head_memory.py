"""What the 8-bit head's calls leave on the device, however many streams they ran on:
the product's status word, and 8 MB at most of workspaces of the rules."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_02438_gb300 import binding, build
    build.build()
    binding.load()
    return binding


def test_rules_keep_no_large_workspace(X):
    x = torch.randn((5000, 257), device="cuda").to(torch.bfloat16)
    am = torch.empty(5000, dtype=torch.int32, device="cuda")
    want = x.float().argmax(dim=1).to(torch.int32)
    streams = [torch.cuda.Stream() for _ in range(8)]
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for st in streams + [torch.cuda.current_stream()]:
        with torch.cuda.stream(st):
            X.process_logits(x, None, am)
        torch.cuda.synchronize()
        assert torch.equal(am, want)
        am.fill_(-9)
        torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() == before


def test_rules_keep_few_small_workspaces(X):
    x = torch.randn((17, 151936), device="cuda").to(torch.bfloat16)
    am = torch.empty(17, dtype=torch.int32, device="cuda")
    want = x.float().argmax(dim=1).to(torch.int32)
    streams = [torch.cuda.Stream(priority=-(i % 2)) for i in range(60)]
    assert len({st.cuda_stream for st in streams}) > 40
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    for _ in range(2):
        for st in streams:
            with torch.cuda.stream(st):
                X.process_logits(x, None, am, rows=17)      # 244800 bytes
            torch.cuda.synchronize()
            assert torch.equal(am, want)
            am.fill_(-9)
            torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before <= 8 << 20
