"""Loads straight to LDS in the generated code: how soon they may follow the instructions that set where they write to
and where they read from."""
import os

import pytest

from paper_2509_07103_amd import build, check_codegen

GOOD = """
<kern>:
\ts_mov_b32 m0, s5                        // 000000001000
\ts_nop 0                                 // 000000001004
\tglobal_load_lds_dwordx4 v3, s[72:73]    // 000000001008
\tv_readfirstlane_b32 s72, v9             // 000000001010
<L0>:
\ts_mov_b32 m0, s6                        // 000000001014
\ts_nop 4                                 // 000000001018
\tglobal_load_lds_dword v3, s[72:73]      // 00000000101C
\ts_cbranch_scc1 L0                       // 000000001024
\ts_endpgm                                // 000000001028
"""


def test_accepts_loads_that_wait():
    assert check_codegen.check_lds_load_waits(GOOD) == {"kern": 2}


@pytest.mark.parametrize("old,new", [
    ("\ts_nop 0                                 // 000000001004\n", ""),                       # straight after m0
    ("\ts_nop 4", "\ts_nop 2"),                                                             # four states after a vector write
    ("\ts_nop 4", "\tv_readlane_b32 s73, v1, 3"),
    ("\ts_nop 4", "\tv_add_co_u32_e64 v4, s[72:73], v4, v5"),                               # its second result
    ("\ts_mov_b32 m0, s6                        // 000000001014\n\ts_nop 4", "\ts_nop 1"),   # two, through the fall into the loop
])
def test_rejects_loads_that_come_too_soon(old, new):
    assert old in GOOD
    with pytest.raises(RuntimeError, match="too soon"):
        check_codegen.check_lds_load_waits(GOOD.replace(old, new))


def test_follows_jumps():
    """The path round a loop: the vector write stands after the load."""
    text = GOOD.replace("\tv_readfirstlane_b32 s72, v9             // 000000001010\n", "")
    assert check_codegen.check_lds_load_waits(text)["kern"] == 2
    late = text.replace("\ts_cbranch_scc1", "\tv_readfirstlane_b32 s72, v9\n\ts_cbranch_scc1").replace("\ts_nop 4", "\ts_nop 1")
    with pytest.raises(RuntimeError, match="too soon"):
        check_codegen.check_lds_load_waits(late)


def test_no_load_of_the_library_comes_too_soon():
    if not os.path.exists(build.LIB):
        build.build()
    counts = check_codegen.check_lds_loads()
    assert any("product_kernel" in k for k in counts) and any("linear_kernel" in k for k in counts)
