"""A call on a stream given by handle writes memory that the current stream just freed: it
waits for the current stream's work, which still reads it."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("default", [False, True])
def test_memory_freed_on_the_current_stream(default):
    import torch

    import paper_2506_02475_amd as comba

    print("stream handle: freed memory, default", default, flush=True)
    T, D = 4096, 1024
    here, side = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.randn(1, T, D, device="cuda").bfloat16()
    w, m = torch.randn(D, 4, device="cuda"), torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(here):
        held = torch.ones_like(x)
        for _ in range(10):  # some milliseconds in front of the read
            m = m @ m * 1e-4
        seen = held + 0
        del held
        y, _ = comba.comba_conv_fwd(x, w, stream=0 if default else side.cuda_stream,
                                    output_final_state=False)
    torch.cuda.synchronize()
    assert (seen == 1).all()
    assert torch.equal(y, comba.comba_conv_fwd(x, w)[0])
