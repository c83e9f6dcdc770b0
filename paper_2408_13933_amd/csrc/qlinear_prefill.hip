// Prefill-shaped qlinear: the launches of the tiled int8 MFMA GEMM of
// qlinear_tiles.h with the requant epilogue.
#include "qlinear_tiles.h"

namespace mq {
namespace {

template <class C, bool ASYM>
__global__ __launch_bounds__(C::THREADS, C::OCC) void qlinear_prefill_kernel(QLinearArgs p,
                                                                       int tiles_n, int tiles_m,
                                                                       int splits,
                                                                       int kt_per_split)
{
    prefill_body<C, ASYM, false>(p, nullptr, tiles_n, tiles_m, splits, kt_per_split);
}

// the dequantized outputs (fp32) written by the epilogue, the codes too
// when p.y is set
template <class C, bool ASYM>
__global__ __launch_bounds__(C::THREADS, C::OCC) void qlinear_prefill_dequant_kernel(
    QLinearArgs p, int tiles_n, int tiles_m, int splits, int kt_per_split)
{
    prefill_body<C, ASYM, false, true>(p, nullptr, tiles_n, tiles_m, splits, kt_per_split);
}

// several linears on one input, without a K split (kt: K stages)
template <class C, bool ASYM>
__global__ __launch_bounds__(C::THREADS, C::OCC) void qlinear_prefill_group_kernel(
    QLinearArgs p, GroupArgs g, int tiles_n, int tiles_m, int kt)
{
    prefill_body<C, ASYM, true>(p, &g, tiles_n, tiles_m, 1, kt);
}

template <class C, bool ASYM>
hipError_t launch_cfg(const QLinearArgs& p, int splits, hipStream_t s)
{
    const int64_t tiles_n = (p.N + C::TN - 1) / C::TN;
    const int64_t tiles_m = (p.M + C::TM - 1) / C::TM;
    const int64_t total = tiles_n * tiles_m;
    const int64_t kt = (p.K + C::BK - 1) / C::BK;
    const int64_t kt_per_split = (kt + splits - 1) / splits;
    splits = (int)((kt + kt_per_split - 1) / kt_per_split);  // every slice non-empty
    if (total * splits > 0x7FFFFFFF || p.batch > 65535) return hipErrorInvalidValue;
    // more than 64 KiB of dynamic LDS must be opted into once per kernel
    constexpr int lds = ASYM || C::A16 ? C::LDS_ASYM : C::LDS;
    const dim3 grid((unsigned)(total * splits), (unsigned)p.batch);
    if constexpr (!C::A16) {
        if (p.y_f) {
            static const hipError_t attr_f = hipFuncSetAttribute(
                reinterpret_cast<const void*>(&qlinear_prefill_dequant_kernel<C, ASYM>),
                hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (attr_f != hipSuccess) return attr_f;
            qlinear_prefill_dequant_kernel<C, ASYM><<<grid, dim3(C::THREADS), lds, s>>>(
                p, (int)tiles_n, (int)tiles_m, splits, (int)kt_per_split);
            return hipGetLastError();
        }
    }
    static const hipError_t attr = hipFuncSetAttribute(
        reinterpret_cast<const void*>(&qlinear_prefill_kernel<C, ASYM>),
        hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    qlinear_prefill_kernel<C, ASYM><<<grid, dim3(C::THREADS), lds, s>>>(
        p, (int)tiles_n, (int)tiles_m, splits, (int)kt_per_split);
    return hipGetLastError();
}

template <class C, bool ASYM>
hipError_t launch_group_cfg(const QLinearArgs& p, GroupArgs g, hipStream_t s)
{
    const int64_t tiles_m = (p.M + C::TM - 1) / C::TM;
    int64_t cols = 0;
    for (int i = 0; i < g.n; ++i) {
        g.part[i].tile0 = (int32_t)(cols * tiles_m);
        g.part[i].tiles_n = (int32_t)((g.part[i].N + C::TN - 1) / C::TN);
        cols += g.part[i].tiles_n;
        if (cols * tiles_m > 0x7FFFFFFF) return hipErrorInvalidValue;
    }
    const int64_t kt = (p.K + C::BK - 1) / C::BK;
    constexpr int lds = ASYM ? C::LDS_ASYM : C::LDS;
    static const hipError_t attr = hipFuncSetAttribute(
        reinterpret_cast<const void*>(&qlinear_prefill_group_kernel<C, ASYM>),
        hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    qlinear_prefill_group_kernel<C, ASYM><<<dim3((unsigned)(cols * tiles_m)), dim3(C::THREADS),
                                            lds, s>>>(p, g, (int)cols, (int)tiles_m, (int)kt);
    return hipGetLastError();
}

template <int WB, int OB, bool ASYM>
hipError_t launch_a(const QLinearArgs& p, hipStream_t s)
{
    Choice ch = choose(p, p.ws != nullptr);
    if (ch.splits > 1 && workspace_for(p, ch) > p.ws_bytes) ch = choose(p, false);
    switch (ch.tile) {
    case kTile256x128: return launch_cfg<T256x128<WB, OB>, ASYM>(p, ch.splits, s);
    case kTile192x256: return launch_cfg<T192x256<WB, OB>, ASYM>(p, ch.splits, s);
    case kTile64x64: return launch_cfg<T64x64<WB, OB>, ASYM>(p, ch.splits, s);
    case kTile256x256W8: return launch_cfg<T256x256W8<WB, OB>, ASYM>(p, ch.splits, s);
    case kTile64x128: return launch_cfg<T64x128<WB, OB>, ASYM>(p, ch.splits, s);
    default: return launch_cfg<T128x128<WB, OB>, ASYM>(p, ch.splits, s);
    }
}

template <int WB, int OB>
hipError_t launch_t(const QLinearArgs& p, hipStream_t s)
{
    return p.w_zp ? launch_a<WB, OB, true>(p, s) : launch_a<WB, OB, false>(p, s);
}

template <int WB, int OB, bool ASYM>
hipError_t launch_group_a(const QLinearArgs& p, const GroupArgs& g, hipStream_t s)
{
    int64_t Ns[kMaxGroup];
    for (int i = 0; i < g.n; ++i) Ns[i] = g.part[i].N;
    const Choice ch = choose(p, false, Ns, g.n);
    switch (ch.tile) {
    case kTile256x128: return launch_group_cfg<T256x128<WB, OB>, ASYM>(p, g, s);
    case kTile192x256: return launch_group_cfg<T192x256<WB, OB>, ASYM>(p, g, s);
    case kTile64x64: return launch_group_cfg<T64x64<WB, OB>, ASYM>(p, g, s);
    case kTile256x256W8: return launch_group_cfg<T256x256W8<WB, OB>, ASYM>(p, g, s);
    case kTile64x128: return launch_group_cfg<T64x128<WB, OB>, ASYM>(p, g, s);
    default: return launch_group_cfg<T128x128<WB, OB>, ASYM>(p, g, s);
    }
}

template <int WB, int OB>
hipError_t launch_group_t(const QLinearArgs& p, const GroupArgs& g, hipStream_t s)
{
    return p.w_zp ? launch_group_a<WB, OB, true>(p, g, s)
                  : launch_group_a<WB, OB, false>(p, g, s);
}

}  // namespace

bool prefill_supported(const QLinearArgs& p)
{
    const int64_t ab = p.a_bits / 8, ob = p.out_bits / 8;
    const int64_t lda = eff_lda(p) * ab, ldy = eff_ldy(p) * ob;
    const int64_t ldw = p.w_bits == 8 ? eff_ldw(p) : (p.ldw ? p.ldw : p.K / 2);
    // whole 16-byte chunks per row (packed int4 rows too), 16-byte aligned
    // rows and batches; output rows of any length and alignment
    const bool kok = p.w_bits == 8 ? (p.K % 16 == 0) : (p.K % 32 == 0);
    const bool align = ((uintptr_t)p.a % 16) == 0 && ((uintptr_t)p.w % 16) == 0 &&
                       lda % 16 == 0 && ldw % 16 == 0 && (p.a_bs * ab) % 16 == 0 &&
                       p.w_bs % 16 == 0;
    // byte offsets inside one 256-row tile must fit the 32-bit buffer offset
    const int64_t lim = (int64_t)1 << 31;
    const bool nok = 256 * ldy < lim && 256 * lda < lim && 256 * ldw < lim &&
                     (!p.y_f || 256 * p.N * 4 < lim);
    // 16-bit activation codes: int8 weights only (the W8A16 tile), which
    // also takes strides, batches and int64 row terms; the 8-bit tiles take
    // dense single products
    const bool dense = p.lda == 0 && p.ldw == 0 && p.ldy == 0 && p.batch == 1 &&
                       p.row_off == nullptr && p.ws_stride == 1;
    const bool aok = p.a_bits == 8 ? dense : (p.w_bits == 8 && p.w_zp == nullptr);
    return kok && align && nok && aok && p.batch >= 1 && p.batch <= 65535;
}

int64_t prefill_workspace_bytes(const QLinearArgs& p)
{
    return workspace_for(p, choose(p, true));
}

int64_t prefill_counter_bytes(const QLinearArgs& p)
{
    const Choice ch = choose(p, true);
    if (ch.splits <= 1) return 0;
    const TileModel& t = kTiles[ch.tile];
    return split_counter_bytes(((p.M + t.tm - 1) / t.tm) * ((p.N + t.tn - 1) / t.tn));
}

// 16-bit activation codes: no K split; ASYM: int64 row terms.  Layers (one
// dense product, no row terms) take the tile of the time model; batched,
// strided and causal products 64x64 up to 64 channels and 128x128 above, the
// tiles their causal column sums are laid out for.
template <int>
hipError_t launch_a16(const QLinearArgs& p, hipStream_t s)
{
    const bool ro = p.row_off != nullptr, o8 = p.out_bits == 8;
    if (p.K <= T128x128A16S2<8>::A16_I32_MAX_K && p.bias == nullptr) {
        if (ro) return o8 ? launch_cfg<T128x128A16S2<8>, true>(p, 1, s)
                          : launch_cfg<T128x128A16S2<16>, true>(p, 1, s);
        return o8 ? launch_cfg<T128x128A16S2<8>, false>(p, 1, s)
                  : launch_cfg<T128x128A16S2<16>, false>(p, 1, s);
    }
    const bool layer = !ro && p.batch == 1 && p.lda == 0 && p.ldw == 0 && p.ldy == 0 &&
                       p.out_causal < 0 && p.in_causal < 0;
    const int tile = layer ? choose_a16(p) : p.N <= 64 ? kA16T64x64 : kA16T128x128;
    if (tile == kA16T64x128)
        return o8 ? launch_cfg<T64x128A16<8>, false>(p, 1, s)
                  : launch_cfg<T64x128A16<16>, false>(p, 1, s);
    if (tile == kA16T128x192)
        return o8 ? launch_cfg<T128x192A16<8>, false>(p, 1, s)
                  : launch_cfg<T128x192A16<16>, false>(p, 1, s);
    if (tile == kA16T64x64) {
        if (ro) return o8 ? launch_cfg<T64x64A16<8>, true>(p, 1, s)
                          : launch_cfg<T64x64A16<16>, true>(p, 1, s);
        return o8 ? launch_cfg<T64x64A16<8>, false>(p, 1, s)
                  : launch_cfg<T64x64A16<16>, false>(p, 1, s);
    }
    if (ro) return o8 ? launch_cfg<T128x128A16<8>, true>(p, 1, s)
                      : launch_cfg<T128x128A16<16>, true>(p, 1, s);
    return o8 ? launch_cfg<T128x128A16<8>, false>(p, 1, s)
              : launch_cfg<T128x128A16<16>, false>(p, 1, s);
}

hipError_t launch_qlinear_prefill_group(const QLinearArgs& p, GroupArgs g, hipStream_t s)
{
    if (p.a_bits != 8 || g.n < 1 || g.n > kMaxGroup) return hipErrorInvalidValue;
    if (p.w_bits == 8 && p.out_bits == 8) return launch_group_t<8, 8>(p, g, s);
    if (p.w_bits == 8) return launch_group_t<8, 16>(p, g, s);
    if (p.out_bits == 8) return launch_group_t<4, 8>(p, g, s);
    return launch_group_t<4, 16>(p, g, s);
}

hipError_t launch_qlinear_prefill(const QLinearArgs& p, hipStream_t s)
{
    if (p.a_bits == 16) return launch_a16<8>(p, s);
    if (p.w_bits == 8 && p.out_bits == 8) return launch_t<8, 8>(p, s);
    if (p.w_bits == 8) return launch_t<8, 16>(p, s);
    if (p.out_bits == 8) return launch_t<4, 8>(p, s);
    return launch_t<4, 16>(p, s);
}

}  // namespace mq
