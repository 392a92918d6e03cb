"""A launch that fails is told to the caller, whichever launch of whichever call it is."""
from paper_2608_08020_gb300 import binding as B
from tests.host_only import CALLS, host_only  # noqa: F401

EACH = CALLS + """
out = []
for dtype in (B.GB_F32, B.GB_BF16, B.GB_FP8):
    n = sum(1 for _ in calls(0))
    for which in range(n):
        at = 0
        while True:                       # the call with its launch number `at` failing, after good ones
            p = pool(dtype)
            for i, (name, f) in enumerate(calls(p)):
                if i == which:
                    fake.fake_fail_at(at)
                    got, text = code(f)
                    done = fake.fake_calls()
                    fake.fake_fail_at(-1)
                    break
                assert code(f) == (0, ""), name
            out.append((dtype, name, at, done, got))
            if done <= at:
                break
            at += 1
print(json.dumps(out))
"""

REGISTERS = CALLS + """
p = pool(B.GB_FP8)
B.gb_pool_seed(p, 2, 20, AT, AT, 0)
fake.fake_regs(160)
few = code(lambda: B.gb_decode_attention(p, 0, AT, AT, AT, 0.1, AT, 0, 0))
print(json.dumps(few))
"""


def test_each_launch_that_fails(host_only):  # noqa: F811
    results = host_only(EACH)
    assert len({(d, name) for d, name, *_ in results}) == 3 * 23
    for dtype, name, at, done, got in results:
        want = B.GB_ERR_CUDA if at < done else B.GB_OK   # (the last time round nothing fails)
        assert got == want, f"type {dtype}: {name}, launch {at} of {done}"


def test_too_few_registers_at_launch(host_only):  # noqa: F811
    """The 8-bit attention's warps share out more registers than a smaller build would launch with."""
    got, text = host_only(REGISTERS)
    assert got == B.GB_ERR_CUDA and "decode" in text
