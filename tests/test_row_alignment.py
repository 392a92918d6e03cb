"""Rows that do not start on 16 bytes are refused by every call that takes rows, before it launches anything: the kernels read them in
pieces of 16 bytes."""
from paper_2608_08020_gb300 import binding as B
from tests.host_only import CALLS, host_only  # noqa: F401

SCRIPT = CALLS + """
out = []
for dtype in (B.GB_F32, B.GB_BF16, B.GB_FP8):
    for off in (2, 4, 8):
        p, bad = pool(dtype), AT + off
        fake.fake_fail_at(-1)
        for k, v in ((bad, AT), (AT, bad)):
            out.append(code(lambda: B.gb_pool_seed(p, 2, 20, k, v, 0)))
        assert fake.fake_calls() == 0
        B.gb_pool_seed(p, 2, 20, AT, AT, 0)
        fake.fake_fail_at(-1)
        for k, v in ((bad, AT), (AT, bad)):
            out.append(code(lambda: B.gb_append_kv(p, 0, 3, k, v, 0)))
            out.append(code(lambda: B.gb_append_kv_rotated(p, 0, 3, ROT, k, v, 0)))
        for q, k, v in ((bad, AT, AT), (AT, bad, AT), (AT, AT, bad)):
            for flags in range(3):
                if q == AT or flags != B.GB_PATH_PER_BEAM or dtype != B.GB_BF16 or off == 2:   # (that one reads q by words)
                    out.append(code(lambda: B.gb_decode_attention(p, 0, q, k, v, 0.1, AT, flags, 0)))
                out.append(code(lambda: B.gb_decode_attention_rotated(p, 0, ROT, q, k, v, 0.1, AT, flags, 0)))
        assert fake.fake_calls() == 0
        for i in range(2):                 # and the pool goes on
            B.gb_append_kv(p, i, 3, AT + 16, AT + 48, 0)
        for i in range(2):
            B.gb_decode_attention(p, i, AT + 16, AT + 32, AT + 48, 0.1, AT + 4, 0, 0)
print(json.dumps(out))
"""


def test_refused(host_only):  # noqa: F811
    out = host_only(SCRIPT)
    assert len(out) == 9 * (2 + 4 + 18) - 2
    for code, text in out:
        assert code == B.GB_ERR_INVALID and "16 bytes" in text
