"""What the kernels of the 4-bit products assume of their LDS, asked of the compiler (no device)."""
import os
import subprocess

from paper_2502_01681_amd import build

SOURCE = """
#include "dg4_mx4.hip"
namespace {
template <typename X> constexpr bool whole_pieces = alignof(X) >= 16 && sizeof(X) % 16 == 0;
template <typename X> constexpr bool rows_apart = sizeof(X) % 16 == 0;
template <int D> constexpr bool layout()
{
    using Rows = MxRows<D>;
    using Store = StoreRows<D>;
    return whole_pieces<Rows> && whole_pieces<MxRows<4 * D>> && whole_pieces<FullRows<float, D>> && whole_pieces<FullRows<bf16_t, D>> && whole_pieces<Store>
        && Rows::STRIDE % 16 == 0 && MxRows<4 * D>::STRIDE % 16 == 0 && rows_apart<decltype(FullRows<float, D>{}.x[0])>
        && rows_apart<decltype(FullRows<bf16_t, D>{}.x[0])> && rows_apart<decltype(Store{}.codes[0])> && sizeof(Store{}.scales[0]) % 8 == 0
        && offsetof(Store, codes) % 16 == 0 && offsetof(Store, scales) % 8 == 0 && offsetof(Rows, codes) % 16 == 0;
}
static_assert(layout<128>() && layout<256>());
}
"""


def test_rows_in_lds_stand_where_16_bytes_can_be_read(tmp_path):
    """They are read and written as pieces of 16 bytes, which the source has to place there: arrays of bytes are not by their type."""
    unit = tmp_path / "layout.hip"
    unit.write_text("#include <cstddef>\n" + SOURCE)
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    got = subprocess.run([hipcc] + build._flags() + ["--cuda-device-only", "-fsyntax-only", "-w", str(unit)], capture_output=True, text=True)
    assert got.returncode == 0, got.stderr[-3000:]
