"""What gb_prompt_attention refuses, before anything is enqueued (no GPU needed: the pointers are never read)."""
import ctypes

import pytest

BASE = dict(q=1 << 20, k=2 << 20, v=3 << 20, out=4 << 20, cu_seqlens=5 << 20, workspace=6 << 20, workspace_bytes=1 << 16,
            q_stride=32 * 128, k_stride=8 * 128, v_stride=8 * 128, out_stride=32 * 128, num_seqs=2, num_tokens=100,
            num_q_heads=32, num_kv_heads=8, head_dim=128, dtype=1, scale=0.1)


def call(**kw):
    from paper_2608_08020_gb300 import binding as B
    if not B.LIB_PATH.exists():
        pytest.skip("libgambit.so not built")
    import torch  # noqa: F401  (loads the CUDA runtime the library links against)
    a = B.GbPromptArgs(**{**BASE, **kw})
    return B.STATUS_NAMES[B.load().gb_prompt_attention(ctypes.byref(a), None)]


@pytest.mark.parametrize("bad,code", [
    (dict(num_q_heads=30), "GB_ERR_INVALID"), (dict(num_q_heads=24), "GB_ERR_UNSUPPORTED"),
    (dict(num_q_heads=0), "GB_ERR_INVALID"), (dict(num_kv_heads=0), "GB_ERR_INVALID"),
    (dict(head_dim=64), "GB_ERR_UNSUPPORTED"), (dict(dtype=0), "GB_ERR_UNSUPPORTED"), (dict(dtype=5), "GB_ERR_INVALID"),
    (dict(num_tokens=-1), "GB_ERR_INVALID"), (dict(num_seqs=-1), "GB_ERR_INVALID"),
    (dict(workspace=0), "GB_ERR_INVALID"), (dict(workspace=(6 << 20) + 16), "GB_ERR_INVALID"),
    (dict(workspace_bytes=0), "GB_ERR_INVALID"), (dict(cu_seqlens=0), "GB_ERR_INVALID"),
    (dict(scale=0.0), "GB_ERR_INVALID"), (dict(scale=-1.0), "GB_ERR_INVALID"), (dict(scale=float("nan")), "GB_ERR_INVALID"),
    (dict(scale=float("inf")), "GB_ERR_INVALID"),
    (dict(q=0), "GB_ERR_INVALID"), (dict(k=0), "GB_ERR_INVALID"), (dict(v=0), "GB_ERR_INVALID"), (dict(out=0), "GB_ERR_INVALID"),
    (dict(q=(1 << 20) + 8), "GB_ERR_INVALID"), (dict(out=(4 << 20) + 2), "GB_ERR_INVALID"),
    (dict(q_stride=32 * 128 - 8), "GB_ERR_INVALID"), (dict(k_stride=8 * 128 + 4), "GB_ERR_INVALID"),
    (dict(v_stride=-1024), "GB_ERR_INVALID"), (dict(out_stride=0), "GB_ERR_INVALID"),
    (dict(out=1 << 20), "GB_ERR_INVALID"), (dict(out=(2 << 20) + 1024), "GB_ERR_INVALID"),
    (dict(num_tokens=2 ** 31 - 1, num_q_heads=128, workspace_bytes=1 << 40), "GB_ERR_TOO_LARGE"),
])
def test_refused(bad, code):
    assert call(**bad) == code


def test_no_tokens_is_no_work():
    assert call(num_tokens=0, q=0, k=0, v=0, out=0) == "GB_OK"


def test_workspace_sizes():
    from paper_2608_08020_gb300 import binding as B
    if not B.LIB_PATH.exists():
        pytest.skip("libgambit.so not built")
    import torch  # noqa: F401
    small = B.gb_prompt_workspace_bytes(0, 0, 8, 8, 128, B.GB_BF16)
    large = B.gb_prompt_workspace_bytes(1 << 20, 4096, 64, 4, 128, B.GB_BF16)
    assert 0 < small <= 512 and small % 256 == 0
    # A unit of 16 bytes for every 8 tokens (128 rows of 16 heads) and every sequence.
    assert large >= 16 * ((1 << 20) // 8 + 4096) and large % 256 == 0
