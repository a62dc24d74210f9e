"""Which forms the exact tests of the learning operators reach, by the library's
own rules (no GPU needed)."""
import ctypes as C

from paper_2407_18352_amd import _abi
from test_dense8_cpu import _compiled

RULES = r"""
#include <cstdio>
#include "f8_rules.hpp"
using namespace hpacml::f8;
int main() {
    long long n, m, k;
    while (std::scanf("%lld %lld %lld", &n, &m, &k) == 3) {
        const Plan p = plan_of(n, m, k);
        std::printf("%d %d %d %lld %u\n", few_rows(n, m, k), p.big, p.parts, (long long)blocks_of(k), p.out_tiles * p.point_tiles);
    }
}
"""


def test_the_exact_tests_reach_the_large_tiles(tmp_path):
    from test_gpu_f8 import PRODUCTS
    from test_gpu_learn_exact import LARGE, LAYERS
    run = _compiled(tmp_path, RULES)

    def plans(shapes):
        lines = run("".join("%d %d %d\n" % s for s in shapes)).split("\n")
        return [tuple(map(int, l.split())) for l in lines[: len(shapes)]]

    got = plans(LARGE)
    big = [(parts, blocks, tiles) for few, large, parts, blocks, tiles in got if large and not few]
    assert any(parts == 1 and tiles > 256 and tiles % 256 for parts, _, tiles in big)          # several a block, not as many for each
    assert any(parts > 1 and blocks % parts for parts, blocks, _ in big) and any(parts > 1 and blocks % parts == 0 for parts, blocks, _ in big)
    assert any(k % 128 == 0 for (_, _, k), g in zip(LARGE, got) if g[1]) and any(k % 128 for (_, _, k), g in zip(LARGE, got) if g[1])
    assert any(not large for _, large, _, _, _ in got)                                         # beside the rule
    small = [g for g in plans(PRODUCTS) if not g[0]]
    assert not any(large for _, large, _, _, _ in small) and {parts > 1 for _, _, parts, _, _ in small} == {False, True}
    y, dx, dw = (plans(s) for s in zip(*[((n, o, i), (n, i, o), (o, i, n)) for n, i, o in LAYERS]))
    assert all({large for _, large, _, _, _ in each} == {0, 1} for each in (y, dx, dw))
    assert max(n for n, _, _ in LAYERS) > 512 * 128                                            # db in two launches


def test_the_exact_tests_reach_every_form_of_group_norm():
    """By the scratch memory: in parts the forward pass needs some; in registers the backward pass needs a row of partial sums for each
    block of the same groups, no more for more images than there are such blocks."""
    from test_gpu_learn_exact import HELD, ONE_POINT, PARTS
    n = C.c_size_t()

    def scratch(kind, backward, images, points, channels, groups):
        assert _abi.lib().hpacmlt_group_norm_scratch(kind, images, points, channels, groups, backward, C.byref(n)) == _abi.OK
        return n.value

    for kind in (_abi.F32, _abi.BF16):
        assert all(scratch(kind, 0, *case) > 0 for case in PARTS)
        assert all(scratch(kind, 0, *case) == 0 for case in HELD)
        for images, *rest in HELD:
            assert scratch(kind, 1, 1, *rest) == 8 * rest[1] < scratch(kind, 1, images - 1, *rest) == scratch(kind, 1, images, *rest)
        in_rows = [case for case in ONE_POINT if scratch(kind, 0, *case) == 0]
        assert len(in_rows) == len(ONE_POINT) - 1                                               # and a group too wide for registers
        again = [scratch(kind, 1, images - 1, *rest) == scratch(kind, 1, images, *rest) for images, *rest in in_rows]
        assert any(again)
