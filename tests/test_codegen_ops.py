"""Waits in the generated code of the operators' kernels (CPU: the built library is
disassembled).

The tile attention asks for the next tile (direct global->LDS loads), the next mask
bytes and the next queries under the products of the current tile, and waits for all of
them once, at the end of the tile.  A wait that the compiler adds before the tile's last
LDS read would drain them where they are asked for.
"""
import re

import pytest

from test_codegen import _is_mfma, _is_register_load, _named, _waits_for_loads, kernels  # noqa: F401


def _is_direct_load(i):
    return re.match(r"(global|buffer)_load", i) and re.search(r"\blds\b", i)


@pytest.mark.parametrize("head_dim,waves,masked", [(d, w, m) for d in (128, 64, 32) for w in (4, 8) for m in (0, 1)] +
                         [(64, 12, 0), (32, 12, 0)])
def test_tile_attention_waits_once_a_tile(kernels, head_dim, waves, masked):  # noqa: F811
    occ = 3 if waves == 12 else 2
    for name, code in _named(kernels, f"k_xattn_tileILi{head_dim}ELi{waves}ELi{occ}ELb{masked}E").items():
        barriers = [n for n, i in enumerate(code) if i.startswith("s_barrier")]
        assert len(barriers) == 2, name            # the order of the sets; the tiles
        tile = code[barriers[-1]:]
        reads = [n for n, i in enumerate(tile) if i.startswith("ds_read_b64_tr_b16")]
        tile = tile[:reads[-1]]
        assert any(map(_is_mfma, tile)) and any(map(_is_direct_load, tile[:reads[0]])), name
        # the next item's queries: their rows' addresses may wait among themselves
        queries = [n for n, i in enumerate(tile) if _is_register_load(i) and "dwordx4" in i]
        assert queries and queries[0] > [n for n, i in enumerate(tile) if _is_direct_load(i)][-1], name
        for n, i in enumerate(tile):
            assert not _waits_for_loads(i) or queries[0] < n < queries[-1], (name, n, i)


@pytest.mark.parametrize("part", ["k_xattn_rowsIDF16b", "k_xattn_rowsIfLi128ELi2E", "k_xattn_split", "k_xattn_f32", "k_xattn_join",
                                  "k_qk_norm"])
def test_few_registers_are_spilled(kernels, part):  # noqa: F811
    for name, code in _named(kernels, part).items():
        spilled = sum(i.startswith("scratch_") for i in code)
        assert spilled <= len(code) // 20, (name, spilled, len(code))
