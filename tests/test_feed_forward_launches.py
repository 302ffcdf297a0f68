"""What the entry points around a feed-forward block's products launch, on a runtime that writes it down in place of a GPU."""
import itertools

import pytest

from paper_2502_08145_amd import binding as B
from tests import host_runtime

A = 1 << 20   # an aligned address; nothing follows it
NN, NT = 0, 1


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    so = host_runtime.build_runtime(tmp_path_factory.mktemp("runtime"))
    return lambda calls: host_runtime.run(so, calls)


def q8_linear(M, N, K):
    return "axonn_q8_linear", [M, N, K, A, A, A, A, A, 0]


def gated_fwd(M, F, D, layout, keep=True):
    return "axonn_gated_fwd", [M, F, D, layout, 0, A, A, A, A if keep else 0, 0]


def launched(answer, what):
    assert answer.status == B.AXONN_OK, what
    assert answer.launches, what
    for x in answer.launches:
        assert 0 < x.workgroups * x.threads < 1 << 32 and x.threads <= 1024 and x.lds <= 160 * 1024, (what, x)


def test_no_size_within_the_limits_is_refused_for_the_kernel_that_was_chosen(run):
    """The kernel that is fastest by its model may not take that many workgroups; then another one runs."""
    rows = [1, 2, 4, 8, 16, 32, 33, 1000, 1 << 20, 1 << 22, 1 << 26, (1 << 26) + 1, 1 << 28, 1 << 30]
    sizes = [s for s in itertools.product(rows, rows, [1, 128, 512, 8192, 1 << 24]) if max(s[0] * s[1], s[0] * s[2], s[1] * s[2]) < 1 << 40
             and -(-s[0] // 256) * -(-s[1] // 256) < 1 << 22]
    for s, answer in zip(sizes, run([q8_linear(*s) for s in sizes])):
        launched(answer, s)

    rows = [1, 3, 5, 16, 72, 1000, 1 << 20, 1 << 22, 1 << 26, (1 << 29) + 3, (1 << 30) - 1]
    sizes = [s for s in itertools.product(rows, rows, [1, 7, 8, 136, 8192, 1 << 24, (1 << 30) - 1], [NN, NT])
             if max(s[0] * s[2], 2 * s[1] * s[2], 2 * s[0] * s[1]) < 1 << 40]
    for s, answer in zip(sizes, run([gated_fwd(*s) for s in sizes])):
        launched(answer, s)


def test_sizes_beyond_the_limits_are_refused(run):
    assert [a.status for a in run([q8_linear(1 << 20, (1 << 20) - 1, 128)])] == [B.AXONN_ERR_UNSUPPORTED]
    assert [a.status for a in run([gated_fwd(1 << 30, 8, 8, NN), gated_fwd(1 << 20, 1 << 19, 8, NT)])] == [B.AXONN_ERR_INVALID_ARG] * 2


@pytest.mark.parametrize("M, F, D, layout", [(130, (1 << 28) + 70, 1, NT), ((1 << 29) + 3, 3, 8, NN)])
def test_the_general_kernel_in_several_launches_covers_its_output_once(run, M, F, D, layout):
    answer, = run([gated_fwd(M, F, D, layout)])
    assert len(answer.launches) > 1 and all("gated_any_kernel" in x.kernel for x in answer.launches)
    assert sum(x.workgroups for x in answer.launches) == -(-M // 64) * -(-F // 64)


FIRST_CALLS = [q8_linear(8192, 8192, 256), q8_linear(2048, 4096, 16384), q8_linear(1000, 1000, 256), q8_linear(64, 64, 256), gated_fwd(2048, 8192, 4096, NN), gated_fwd(2048, 8192, 4096, NT),
               gated_fwd(299, 2088, 1608, NN), gated_fwd(300, 2048, 128, NT), gated_fwd(16, 8192, 4096, NT), gated_fwd(40, 501, 777, NN),
               ("axonn_linear_fwd", [2048, 4096, 4096, NN, A, A, A, 1, 0])]


@pytest.mark.parametrize("call", FIRST_CALLS)
def test_lds_limits_are_raised_by_the_set_up_or_by_the_first_call(run, call):
    init, first = run([("axonn_linear_init", []), call])
    assert init.status == B.AXONN_OK and first.status == B.AXONN_OK and first.launches
    assert not first.limits, "the set-up left these to the call"
    raised = dict(init.limits)
    for x in first.launches:
        assert x.lds <= 64 * 1024 or raised[x.kernel] >= x.lds, x
    first, second = run([call, call])
    raised = dict(first.limits)
    assert not second.limits and first.launches == second.launches
    for x in first.launches:
        assert x.lds <= 64 * 1024 or raised[x.kernel] >= x.lds, x


def test_no_dynamic_lds_is_used_without_its_limit(run):
    """Over many sizes: every launch stays within what its kernel's limit was raised to."""
    sizes = list(itertools.product([1, 5, 16, 17, 40, 64, 130, 300, 520, 2048], [16, 72, 200, 501, 2048, 4099, 8192], [64, 136, 777, 4096]))
    answers = run([("axonn_linear_init", [])] + [q8_linear(*s) for s in sizes] + [gated_fwd(*s, layout) for s in sizes for layout in (NN, NT)])
    raised = dict(answers[0].limits)
    for answer in answers[1:]:
        for x in answer.launches:
            assert x.lds <= 64 * 1024 or raised.get(x.kernel, 0) >= x.lds, x


def test_scratch_memory_is_a_tensor():
    """An address has no size: it is refused as any other that is no tensor."""
    with pytest.raises(TypeError):
        B.axonn_rmsnorm_bwd(8, 8, A, A, A, A, None, A, A, A, stream=0)
    with pytest.raises(TypeError):
        B.axonn_gated_bwd_q8(8, 8, 8, "NN", "silu", A, A, A, A, A, A, A, A, A, A, A, stream=0)
