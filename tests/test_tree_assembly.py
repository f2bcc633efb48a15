"""The attention of trees keeps its copies in flight as the one over shared prefixes does: its loops over tiles that need no mask neither wait for
vector memory by themselves nor spill registers."""
import os

import pytest

import paper_2511_07423_amd as synera
from test_shared_assembly import whole_loops

ASM = os.path.join(os.path.dirname(synera.lib_path()), "_build", "tree-hip-amdgcn-amd-amdhsa-gfx950.s")


@pytest.mark.parametrize("head_dim", [64, 128])
def test_each_form_of_the_attention_has_its_loop(head_dim):
    """Four wavefronts to the keys (no barrier), two by two (one), four to the rows (one for two tiles)."""
    if not os.path.exists(ASM):
        pytest.skip("the library was built elsewhere: no assembly here")
    marked, spans = whole_loops(open(ASM).read(), rf"_Z16tree_attn_kernelILi{head_dim}EEv12TreeAttnArgs")
    tile = head_dim // 8                          # products of a tile: head_dim / 16 of the scores, 2 x head_dim / 32 of the values

    def count(span, word):
        return sum(word in x for x, _ in marked[span[0]: span[1] + 1])
    by_key = [s for s in spans if count(s, "v_mfma") and not count(s, "global_load_lds")]
    free = [s for s in spans if count(s, "v_mfma") in (tile, 2 * tile) and count(s, "global_load_lds") and
            not any(s[0] <= k[0] and k[1] <= s[1] for k in by_key)]
    free = [s for s in free if not any(o[0] <= s[0] and s[1] <= o[1] and o != s for o in free)]
    assert sorted((count(s, "v_mfma") // tile, count(s, "s_barrier")) for s in free) == [(1, 0), (1, 1), (2, 1)]
    for a, b in free:
        spills = [x for x, _ in marked[a: b + 1] if "scratch_" in x]
        waits = [x for x, inline in marked[a: b + 1] if "s_waitcnt" in x and "vmcnt" in x and not inline]
        assert not spills and not waits, (spills[:3], waits[:3])
