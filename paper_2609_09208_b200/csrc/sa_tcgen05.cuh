// The tensor cores of sm_100a by way of tensor memory: allocation, descriptors, products and the way into and out of registers.
//
// Operands in shared memory are rows of 128 bytes, 64 numbers of 16 bits, in blocks of 8 rows (1024 bytes, 1024-byte aligned), the 16-byte
// pieces of row r at places piece ^ (r % 8): the 128-byte swizzle.  An operand whose rows run along the contraction (queries, keys) and one whose
// rows run across it (values: a row is a key's 64 channels) are laid out alike; the instruction descriptor says which.
#pragma once
#include "sa_common.cuh"
#include "sa_stage.cuh"

namespace sa {

constexpr uint32_t kTmemColumns = 512;

// By one warp; `at`: shared address of the word that receives the address of the first column: 0, as all columns are asked for.
SA_D void tmem_alloc(uint32_t at) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(at), "r"(kTmemColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
SA_D void tmem_free() { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(0u), "r"(kTmemColumns) : "memory"); }

// One lane of the warp; the others' instructions below are issued with `go` false.  So the warp stays together, and operands that are the same for all lanes stay
// in its uniform registers, from where these instructions take them (in a branch of one lane every operand was moved there, 70 cycles a product).
SA_D bool elect_lane() {
    uint32_t x;
    asm volatile("{.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;}" : "=r"(x));
    return x != 0;
}

SA_D void tcgen05_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
SA_D void tcgen05_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// One arrival at the mbarrier once all products that this thread has issued are done.
SA_D void tcgen05_commit(uint32_t mbar, bool go) {
    asm volatile("{.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];}" ::"r"(mbar), "r"((uint32_t)go) : "memory");
}

// Shared-memory operand at `at` (see above), the lower word of its descriptor: blocks of 64 numbers across the contraction `across` bytes apart.  Its upper word says that blocks of
// 8 rows are 1024 bytes apart.  An operand `n` bytes further on is n / 16 more.
SA_D uint32_t smem_operand(uint32_t at, uint32_t across = 1024) { return (at >> 4) | (across >> 4) << 16; }
constexpr uint32_t kOperandUpper = (1024u >> 4) | 1u << 14 | 2u << 29;
// 128 x N products of 16-bit numbers (BF16: bfloat16, else binary16), FP32 sums; the second operand's rows run across the contraction.
SA_HD constexpr uint32_t mma_form(int n, bool bf16, bool b_across) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (b_across ? 1u : 0u) << 16 | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}
// 16 numbers of the contraction; add: to the sums that are there.
SA_D void tcgen05_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t form, bool add, bool go) {
    asm volatile("{.reg .pred p, q;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b64 a, {%1, %6};\n\tmov.b64 b, {%2, %6};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;}" ::"r"(d), "r"(a), "r"(b), "r"(form), "r"((uint32_t)add), "r"((uint32_t)go), "r"(kOperandUpper)
                 : "memory");
}
// ... with the first operand in tensor memory, two numbers a column.
SA_D void tcgen05_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t form, bool add, bool go) {
    asm volatile("{.reg .pred p, q;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\tmov.b64 b, {%2, %6};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;}" ::"r"(d), "r"(a), "r"(b), "r"(form), "r"((uint32_t)add), "r"((uint32_t)go), "r"(kOperandUpper)
                 : "memory");
}

// 32 (16) columns of this warp's 32 rows, a row a thread.  The registers are there after tmem_loaded().
SA_D void tmem_load(uint32_t at, uint32_t (&x)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]),
          "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(x[16]), "=r"(x[17]), "=r"(x[18]), "=r"(x[19]), "=r"(x[20]),
          "=r"(x[21]), "=r"(x[22]), "=r"(x[23]), "=r"(x[24]), "=r"(x[25]), "=r"(x[26]), "=r"(x[27]), "=r"(x[28]), "=r"(x[29]), "=r"(x[30]), "=r"(x[31])
        : "r"(at));
}
SA_D void tmem_load(uint32_t at, uint32_t (&x)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]),
          "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
        : "r"(at));
}
SA_D void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
SA_D void tmem_store(uint32_t at, const uint32_t (&x)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(x[0]),
        "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]),
        "r"(x[16]), "r"(x[17]), "r"(x[18]), "r"(x[19]), "r"(x[20]), "r"(x[21]), "r"(x[22]), "r"(x[23]), "r"(x[24]), "r"(x[25]), "r"(x[26]), "r"(x[27]), "r"(x[28]), "r"(x[29]), "r"(x[30]),
        "r"(x[31]), "r"(at)
        : "memory");
}
SA_D void tmem_store(uint32_t at, const uint32_t (&x)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(x[0]),
        "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]), "r"(at)
        : "memory");
}
SA_D void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

}  // namespace sa
