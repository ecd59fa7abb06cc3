"""Launch plans of the attention on a clean region in 4 bits (attend_split.hpp), compiled for the CPU: no GPU needed."""
import ctypes
import random
import subprocess

import pytest

from paper_2602_10825_amd import build

DRIVER = r"""
#include "attend_split.hpp"
static FcAttendPlan plan(int f32, int A, int L_c, int L_clean, int H_q, int d, int may_split) {
    return f32 ? fc_attend_plan_kv4_f32(A, L_c, L_clean, H_q, d, may_split) : fc_attend_plan_kv4(A, L_c, L_clean, H_q, d, may_split);
}
extern "C" {
// partials that the plans ask for, the most over key counts from 0 to 2^17
__attribute__((visibility("default"))) int parts(int f32, int A, int L_c, int H_q, int d) {
    int most = 0;
    for (int clean = 0; clean < 1 << 17; clean += 1 + clean / 7) {
        const int b = plan(f32, A, L_c, clean, H_q, d, 1).parts;
        most = most > b ? most : b;
    }
    return most;
}
__attribute__((visibility("default"))) int undivided(int f32, int A, int L_c, int L_clean, int H_q, int d) {
    const FcAttendPlan p = plan(f32, A, L_c, L_clean, H_q, d, 0);
    int most = p.parts + p.merge_grid;
    for (int R = 0; R < A; ++R) most += p.splits[R] - 1;
    return most;
}
__attribute__((visibility("default"))) int bound(int A, int L_c, int H_q) { return (int)fc_split_parts_bound(A, L_c, H_q); }
}
"""


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, out = d / "plan.hip", d / "plan.so"
    src.write_text(DRIVER)
    subprocess.run([build.HIPCC, "--offload-host-only", *build.FLAGS, "-shared", str(src), "-o", str(out)], check=True)
    return ctypes.CDLL(str(out))


@pytest.mark.parametrize("f32", [0, 1])
def test_workspace_holds_what_any_number_of_keys_can_ask_for(so, f32):
    """A plan beyond it would find no room and leave the keys undivided, several times slower and without an error."""
    rng = random.Random(2)
    for _ in range(2500):
        A, H, d = rng.randint(1, 16), rng.choice((1, 2, 3, 8, 12, 24, 40, 64)), rng.choice((64, 128))
        L_c = int(2 ** rng.uniform(0, 14))
        assert so.parts(f32, A, L_c, H, d) <= so.bound(A, L_c, H), (A, L_c, H, d)


@pytest.mark.parametrize("f32", [0, 1])
def test_without_room_nothing_is_divided(so, f32):
    rng = random.Random(3)
    for _ in range(300):
        args = rng.randint(1, 16), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 17)), rng.choice((1, 2, 12, 24)), rng.choice((64, 128))
        assert so.undivided(f32, *args) == 0, args
