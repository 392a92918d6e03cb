"""The failure path of the prompt and draft pipelines without a fault: a load that never comes, waits that run out.

gb_prompt_wait_selftest leaves one load out and shortens the waits to 50 ms.  The call must end, with every copy and product of
the CTAs that gave up ended before they left, record GB_ERR_TIMEOUT, write no row but right ones, and leave the workspace usable."""
import ctypes
import math
import time

import pytest

from tests.test_gpu_prompt import attend, bound, make

pytestmark = pytest.mark.gpu


class Call:
    def __init__(self, lengths, hq, hkv, seed):
        import torch
        from paper_2608_08020_gb300 import binding as B
        from paper_2608_08020_gb300.prompt import PromptAttention
        self.cu = [0]
        for n in lengths:
            self.cu.append(self.cu[-1] + n)
        self.n, self.scale = self.cu[-1], 1 / math.sqrt(128)
        self.q, self.k, self.v = make("bf16", self.n, hq, hkv, seed)
        self.at = torch.tensor(self.cu, dtype=torch.int32, device="cuda")
        self.op = PromptAttention(hq, hkv, 128, "bf16", max_tokens=self.n, max_seqs=len(lengths))
        self.out = torch.full_like(self.q, 7.0)
        self.args = B.GbPromptArgs(
            q=self.q.data_ptr(), k=self.k.data_ptr(), v=self.v.data_ptr(), out=self.out.data_ptr(), cu_seqlens=self.at.data_ptr(),
            workspace=self.op.workspace.data_ptr(), workspace_bytes=self.op.workspace.numel(), q_stride=hq * 128,
            k_stride=hkv * 128, v_stride=hkv * 128, out_stride=hq * 128, num_seqs=len(lengths), num_tokens=self.n,
            num_q_heads=hq, num_kv_heads=hkv, head_dim=128, dtype=B.GB_BF16, scale=self.scale)
        self.o, self.a = attend(self.q, self.k, self.v, self.cu, self.scale)

    def right(self):
        """Rows (token, head) within the bound."""
        return ((self.out.double() - self.o).abs() <= bound(self.o, self.a, "bf16")).all(-1)


@pytest.mark.parametrize("stalled,at", [(0, 0), (0, 1), (0, 4), (1, 0), (1, 2), (1, 5), (2, 0), (2, 256)])
@pytest.mark.parametrize("lengths,hq,hkv", [([900], 8, 2), ([40, 300, 17, 700, 129, 1300, 64, 500], 32, 8), ([128] * 40 + [1000] * 40, 8, 8)],
                         ids=["one", "packed", "many"])
def test_a_load_that_never_comes(cuda, lengths, hq, hkv, stalled, at):
    import torch
    from paper_2608_08020_gb300 import binding as B
    c = Call(lengths, hq, hkv, seed=31)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    B.gb_prompt_wait_selftest(c.args, stalled, at)
    status = c.op.status()                      # synchronises
    took = time.perf_counter() - t0
    assert status == B.GB_ERR_TIMEOUT
    assert 0.04 < took < 10, took
    left = (c.out == 7).all(-1)
    assert bool((left | c.right()).all()) and bool(left.any())
    c.out.fill_(7.0)
    c.op(c.q, c.k, c.v, c.at, c.scale, c.out)
    assert c.op.status() == B.GB_OK and bool(c.right().all())


def test_nothing_stalled(cuda):
    """A tile that no unit has: the self-test is the call itself."""
    from paper_2608_08020_gb300 import binding as B
    c = Call([300, 200], 8, 2, seed=32)
    for stalled, at in ((0, 3), (1, 3), (2, 7)):
        c.out.fill_(7.0)
        B.gb_prompt_wait_selftest(c.args, stalled, at)
        assert c.op.status() == B.GB_OK and bool(c.right().all())


def test_refusals(cuda):
    from paper_2608_08020_gb300 import binding as B
    c = Call([64], 8, 2, seed=33)
    for stalled, at in ((-1, 0), (3, 0), (0, -1)):
        assert B.load().gb_prompt_wait_selftest(ctypes.byref(c.args), stalled, at, None) == B.GB_ERR_INVALID
    c.args.dtype = B.GB_F32
    assert B.load().gb_prompt_wait_selftest(ctypes.byref(c.args), 0, 0, None) == B.GB_ERR_INVALID
    assert B.load().gb_prompt_wait_selftest(None, 0, 0, None) == B.GB_ERR_INVALID
