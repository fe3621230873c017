"""Which layouts of an output the operators accept: every one whose rows share no element.  Runs on the CPU: each call is
refused, for its layout or, where that is accepted, for its scratch, before anything touches a device."""
import itertools

from paper_2409_09242_amd import binding as B

P = 0x10000              # an address that is never followed
WORKSPACE, ARG = -4, -5


def _status(k, m, n, ld, stride):
    """dw_fp8_matmul with a contraction that needs scratch, and none given."""
    return B.lib().dw_fp8_matmul(P, P, P, P, None, n, k, m, n, 8192, 0, P, ld, stride, None, 0, None)


def _apart(k, m, n, ld, stride):
    at = [w * stride + r * ld + j for w in range(k) for r in range(m) for j in range(n)]
    return len(set(at)) == len(at)


def test_every_layout_of_a_few_rows():
    accepted = 0
    for k, m, n in itertools.product((1, 2, 3, 4), (1, 2, 3, 4), (1, 2, 3)):
        assert B.lib().dw_fp8_matmul_scratch_bytes(k, m, n, 8192) > 0
        for ld, stride in itertools.product(range(0, 11), range(0, 15)):
            # rows of one worker have to follow each other; a stride that is not used may be anything
            want = ARG if (m > 1 and ld < n) or not _apart(k, m, n, ld, stride) else WORKSPACE
            assert _status(k, m, n, ld, stride) == want, (k, m, n, ld, stride)
            accepted += want == WORKSPACE and k > 1 and stride < ld
    assert accepted > 100


def test_larger_layouts():
    for k, m, n, ld, stride, want in (
            (8, 60, 16, 128, 16, WORKSPACE), (8, 60, 16, 127, 16, ARG), (8, 60, 16, 128, 15, ARG), (8, 60, 16, 1 << 40, 16, WORKSPACE),
            (8, 60, 16, 16, 960, WORKSPACE), (8, 60, 16, 16, 959, ARG), (16, 512, 4096, 16 * 4096 - 1, 4096, ARG), (64, 300, 10, 630, 10, ARG),
            (2, 1 << 20, 8, 1 << 20, (1 << 40) - (1 << 20), ARG), (2, 1 << 20, 8, 1 << 20, (1 << 40) - (1 << 20) - 7, ARG)):
        assert want == ARG or B.lib().dw_fp8_matmul_scratch_bytes(k, m, n, 8192) > 0          # (accepted without it would run)
        assert _status(k, m, n, ld, stride) == want, (k, m, n, ld, stride)
