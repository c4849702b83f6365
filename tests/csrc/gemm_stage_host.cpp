// What a stage of a product's loads may reach (csrc/gemm_stage.h) for a host test.
#include "../../paper_2312_08053_amd/csrc/gemm_stage.h"

using namespace kimad;

extern "C" {
uint32_t bytes_of_stage(int across, uint32_t lines, uint32_t count, uint32_t ld_bytes) { return stage_bytes(across, lines, count, ld_bytes); }
uint64_t ld_of(uint64_t rows, uint64_t cols, uint64_t ld) { return stage_ld(rows, cols, ld); }
}
