"""The choice of the matrix product's kernel and its shares of k (csrc/anszp_linear_plan.h), on the host."""
import subprocess

import pytest

from decode_choice import compile_host
from linear_sizes import SIZES

DRIVER = r"""
#include "anszp_linear_plan.h"
#include <cstdio>
int main() {
    static const char* const names[kLinearKernels] = {"any", "few11", "few21", "few22", "few24", "tile64", "tile128", "tile192", "tile256"};
    unsigned long long rows, cols, xs, ws;
    unsigned eight, kb, cus, may;
    while (std::scanf("%u %llu %llu %u %llu %llu %u %u", &eight, &rows, &cols, &kb, &xs, &ws, &cus, &may) == 8) {
        const LinearPlan p = linear_plan(eight != 0, rows, cols, kb, xs, ws, cus, may != 0);
        std::printf("%s %u %u %llu %llu\n", names[p.kernel], p.shares, p.share_steps, (unsigned long long)p.parts_stride, (unsigned long long)p.workspace);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = compile_host(DRIVER, str(tmp_path_factory.mktemp("plan")), "plan")

    def ask(calls):
        """calls: (eight bits, rows, cols, bytes of k, stride of x, of the weights, CUs, may share) each."""
        text = "\n".join(" ".join(str(int(v)) for v in c) for c in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60).stdout.split("\n")
        return [(w[0], *map(int, w[1:])) for w in (line.split() for line in out if line)]

    return ask


def _call(rows, cols, k, eight, cus=256, may=True, stride=0):
    kb = k * (1 if eight else 2)
    return eight, rows, cols, kb, stride or kb, stride or kb, cus, may


def test_every_kernel_is_reached(plan):
    for name, sizes in SIZES.items():
        for got, size in zip(plan([_call(*s) for s in sizes]), sizes):
            assert (got[0] + (" shares" if got[1] > 1 else "")) == name, (size, got)


def test_shares_have_all_of_k_and_room(plan):
    calls = [_call(r, c, k, e, cus, may) for r in (1, 16, 17, 40, 65, 130, 300, 1000, 5000, 20000) for c in (1, 64, 500, 4096, 11008)
             for k in (8, 16, 63, 64, 65, 127, 500, 1000, 4096, 11008, 65536) for e in (False, True) for cus in (64, 256) for may in (False, True)]
    for call, (kernel, shares, steps, stride, workspace) in zip(calls, plan(calls)):
        eight, rows, cols, kb, _, _, _, may = call
        whole = kb // 128
        assert stride == (cols + 7) // 8 * 8
        if shares == 1:
            assert steps == whole and workspace == 0
        else:
            assert may and kernel in ("tile64", "tile128")
            assert shares * steps >= whole > (shares - 1) * steps and steps >= 1          # every share has a step, all together all
            assert workspace == 4 * shares * rows * stride
        if kb < 16:
            assert kernel == "any"
        if rows > 4096:
            assert not kernel.startswith("few")


def test_rows_far_apart(plan):
    """Tiles count bytes behind their first row in 32 bits."""
    for rows in (1, 300, 5000):
        for got in plan([_call(rows, 4096, 4096, False, stride=(1 << 23) + 16)]):
            assert not got[0].startswith("tile")
        for got in plan([_call(5000, 4096, 4096, False, stride=1 << 23)]):
            assert got[0].startswith("tile")


def test_a_launch_has_fewer_than_2_to_the_32_threads(plan):
    """What is beyond is left out without an error.  (The kernel for any sizes has no other to give way to: the call is refused.)"""
    tiles = {"few11": (16, 16, 512), "few21": (32, 16, 512), "few22": (32, 32, 512), "few24": (32, 64, 512), "tile64": (64, 64, 256), "tile128": (128, 128, 256),
             "tile192": (192, 256, 512), "tile256": (256, 256, 512)}
    calls = [_call(r, c, k, e) for r in (1, 16, 33, 300, 4096, 1 << 17, 1 << 21) for c in (1, 4096, 1 << 20, (1 << 26) + 1, (1 << 27) - 15, (1 << 27) + 70, (1 << 28) + 1, (1 << 30) - 63)
             for k in (8, 16, 64) for e in (False, True) if r * c <= 1 << 35]
    for call, got in zip(calls, plan(calls)):
        if got[0] == "any":
            assert call[3] < 16 or call[1] * call[2] > 1 << 34
            continue
        tok, ch, threads = tiles[got[0]]
        across = -(-call[2] // ch)
        assert across * (1 if got[0].startswith("few") else -(-call[1] // tok)) * threads < 1 << 32, (call, got)
