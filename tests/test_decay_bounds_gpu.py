"""Linear attention with a decay per head, on packed sequences whose offsets are wrong: memory
around what a call writes, and the check of a host copy."""
import ctypes

import numpy as np
import pytest

import test_decay_gpu as decay

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class Guarded:
    """Device memory whose surroundings are checked."""
    GUARD, BYTE = 1 << 16, 0xA5

    def __init__(self):
        self.made = []

    def new(self, nbytes):
        import torch

        nbytes = (nbytes + 255) // 256 * 256
        mem = torch.full((nbytes + 2 * self.GUARD,), self.BYTE, dtype=torch.uint8, device="cuda")
        self.made.append(mem)
        return mem.data_ptr() + self.GUARD

    def check(self):
        for i, mem in enumerate(self.made):
            assert bool((mem[:self.GUARD] == self.BYTE).all()), i
            assert bool((mem[-self.GUARD:] == self.BYTE).all()), i


@pytest.mark.parametrize("T,H,Hk", [(192, 2, 1), (1536, 1, 1)], ids=["whole", "cut"])
def test_malformed_device_offsets_write_no_other_memory(T, H, Hk):
    """Offsets that decrease, are negative or lie behind the tokens, without a host copy: what is
    around the outputs and workspaces stays.  (T: a multiple of 64, so that a tensor's guard begins
    at its last byte; the workspaces' begin at the size that the library asks for.)"""
    import torch

    import paper_2506_02475_amd as comba

    lib, S, d = comba.load_library(), 3, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)

    def rnd(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, device="cuda", generator=gen).to(dtype)

    q, k, v, do = rnd(T, H, d), rnd(T, Hk, d), rnd(T, H, d), rnd(T, H, d)
    g, h0 = -torch.rand(T, H, device="cuda", generator=gen), rnd(S, H, d, d, dtype=torch.float32)
    P = torch.Tensor.data_ptr
    for bad in ([-5, 60, 10, 4000], [T, T, 0, 0], [0, 2 ** 31 - 1, -2 ** 31, T], [T, 70, 0, -1],
                [0, T, 0, T], [3, 3, 3, 3]):
        cu = torch.tensor(bad, dtype=torch.int32, device="cuda")
        shp = comba.CombaDecayShape(B=1, T=T, H=H, Hq=H, Hk=Hk, Hv=H, dk=d, dv=d, num_seqs=S,
                                    cu_seqlens=cu.data_ptr(), in_dtype=comba.COMBA_BF16,
                                    g_dtype=comba.COMBA_F32, scale=0.5)
        shp = ctypes.byref(shp)
        m = Guarded()
        save, work = lib.comba_decay_save_bytes(shp), lib.comba_decay_bwd_workspace_bytes(shp)
        o, ht, ws = m.new(T * H * d * 2), m.new(S * H * d * d * 4), m.new(save)
        ins = (P(q), P(k), P(v), P(g), P(h0))
        stream = torch.cuda.current_stream().cuda_stream
        assert lib.comba_decay_fwd_save(shp, *ins, o, ht, ws, save, stream) == 0
        outs = [m.new(n) for n in (T * H * d * 2, T * Hk * d * 2, T * H * d * 2, T * H * 4,
                                   S * H * d * d * 4)]
        ws2 = m.new(work)
        assert lib.comba_decay_bwd(shp, *ins, P(do), None, *outs, ws, save, ws2, work, stream) == 0
        torch.cuda.synchronize()
        m.check()
        del m


def test_offsets_of_a_host_copy_are_checked_before_a_launch():
    import torch

    import paper_2506_02475_amd as comba

    lens = [500, 0, 400, 300]
    c = decay._case("checked", H=1, dk=64, dv=64, lens=lens)
    args = decay._inputs(c)
    cu = np.cumsum([0] + lens).astype(np.int32)
    for bad in ([0, 500, 400, 900, 1200], [0, 500, 500, 900, 1100], [5, 500, 500, 900, 1200]):
        with pytest.raises(comba.CombaError):
            comba.comba_decay_fwd(*args, cu_seqlens=torch.from_numpy(cu).cuda(),
                                  cu_seqlens_host=np.asarray(bad, np.int32))
