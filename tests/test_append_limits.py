"""More tokens than lengths of 32 bits take are refused on the host; as many as they take are the device's to refuse."""
from paper_2608_08020_gb300 import binding as B
from tests.host_only import CALLS, host_only  # noqa: F401

SCRIPT = CALLS + """
out = []
for dtype in (B.GB_F32, B.GB_BF16, B.GB_FP8):
    for n in ((1 << 30) + 1, (1 << 31) - 30, (1 << 31) - 1, 1 << 30):
        p = pool(dtype)
        B.gb_pool_seed(p, 2, 20, AT, AT, 0)
        fake.fake_fail_at(-1)
        got = [code(lambda: B.gb_append_kv(p, 0, n, AT, AT, 0))[0]]
        got += [fake.fake_calls() > 0]
        q = pool(dtype)
        B.gb_pool_seed(q, 2, 20, AT, AT, 0)
        got += [code(lambda: B.gb_append_kv_rotated(q, 0, n, ROT, AT, AT, 0))[0]]
        out.append(got)
print(json.dumps(out))
"""


def test_tokens_of_a_chunk(host_only):  # noqa: F811
    out = host_only(SCRIPT)
    for i, got in enumerate(out):
        assert got == ([B.GB_OK, True, B.GB_OK] if i % 4 == 3 else [B.GB_ERR_INVALID, False, B.GB_ERR_INVALID])
