// Products with 8-bit activations of a scale per token and 8- or 4-bit weights
// of a scale (and zero-point) per channel: exact int32 sums, then
//   y = ((float)sum * w_scale[n]) * a_scale[m] + bias[n]
// in the same fp32 steps on every path, so all paths give the same bits.
//
// One token: the weights are streamed once (memory bounds it), dot4 against the
// token's codes in LDS; where few channels keep the call short, every
// work-group quantizes the token itself and a launch is saved.  2 to 16 tokens:
// the same stream against the 16 columns of an MFMA.  More: the tiles of
// qlinear_tiles.h, bound by the matrix cores, with a floating epilogue.
#include "linear_tokens.h"
#include "qlinear_tiles.h"
#include "wave.h"

namespace mq {
namespace {

constexpr int kStream = 2;  // weights: non-temporal (each byte is read once per call)

__device__ inline void store_out(const TokenArgs& t, int64_t i, float v)
{
    if (t.type == MQ_F32) store_elem<MQ_F32>(t.y, i, v);
    else if (t.type == MQ_BF16) store_elem<MQ_BF16>(t.y, i, v);
    else store_elem<MQ_F16>(t.y, i, v);
}

// ---------------------------------------------------------------------------
// One token.  8 channels per work-group, in each wave load 8 lanes read 128
// bytes of one channel's weights.
constexpr int kChans = 8, kLanes = 64 / kChans;
constexpr int kSteps = 4;  // wave loads in flight per round
constexpr int kHold = 4;   // chunks of 8 activations that a lane holds

struct OneArgs {
    QLinearArgs p;
    TokenArgs t;
    const void* x;  // FUSED: the token's activations
};

// XTYPE: the activations' type where the work-group quantizes them, else -1.
template <int WBITS, int XTYPE, int NW>
__global__ __launch_bounds__(NW * 64) void one_token_kernel(OneArgs a)
{
    constexpr bool FUSED = XTYPE >= 0;
    constexpr int XT = FUSED ? XTYPE : MQ_F32;
    const QLinearArgs& p = a.p;
    extern __shared__ __align__(16) int8_t smem[];
    const int K = (int)p.K;
    int32_t* red = reinterpret_cast<int32_t*>(smem + (K + 15) / 16 * 16);  // [NW][kChans]
    uint32_t* wmax = reinterpret_cast<uint32_t*>(red + NW * kChans);       // [NW]
    int32_t* wsum = reinterpret_cast<int32_t*>(wmax + NW);                 // [NW]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane / kLanes, j = lane % kLanes;
    const int64_t n0 = (int64_t)blockIdx.x * kChans;
    const int wrow = WBITS == 8 ? K : K / 2;
    const int rows = (int)(p.N - n0 < kChans ? p.N - n0 : kChans);
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(static_cast<const int8_t*>(p.w) + n0 * wrow), (short)0, rows * wrow, 0x00020000);

    // the activations first: the weights behind them need no answer before
    Raw<XT, 8> xr[FUSED ? kHold : 1];
    constexpr int E = XT == MQ_F32 ? 4 : 2;
    if constexpr (FUSED) {
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            const int k = (i * NW * 64 + tid) * 8;
            if (k < K) xr[i].load(static_cast<const int8_t*>(a.x) + k * E);
        }
    }
    const bool epi = wave == 0 && lane < kChans;
    float ws = 0.0f, bias = -0.0f, scale = 0.0f;
    int32_t zw = 0, rs = 0;
    if (epi) {
        const int64_t n = n0 + lane < p.N ? n0 + lane : p.N - 1;
        ws = p.w_scale[n];
        if (p.bias) bias = p.bias[n];
        if (p.w_zp) zw = p.w_zp[n];
        if constexpr (!FUSED) {
            scale = a.t.scale[0];
            if (p.w_zp) rs = p.a_rowsum[0];
        }
    }
    const int steps = (wrow + kLanes * 16 - 1) / (kLanes * 16);
    const int s_begin = steps * wave / NW, s_end = steps * (wave + 1) / NW;
    v4i wv[kSteps];
    auto load = [&](int s) {
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int off = ((s + u) * kLanes + j) * 16;
            const uint32_t dead = (uint32_t)((s + u >= s_end) | (off >= wrow)) << 31;
            wv[u] = __builtin_amdgcn_raw_buffer_load_b128(rw, (uint32_t)(c * wrow + off) | dead, 0,
                                                          kStream);
        }
    };
    if constexpr (!FUSED) {
        load(s_begin);
        const __amdgpu_buffer_rsrc_t ra =
            __builtin_amdgcn_make_buffer_rsrc((void*)p.a, (short)0, K, 0x00020000);
        for (int i = tid; i < K / 16; i += NW * 64)
            *reinterpret_cast<v4i*>(smem + i * 16) =
                __builtin_amdgcn_raw_buffer_load_b128(ra, (uint32_t)(i * 16), 0, 0);
    } else {
        load(s_begin);
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < kHold; ++i)
            if ((i * NW * 64 + tid) * 8 < K)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = max(most, abs_bits(xr[i][e]));
        most = wave_max(most);
        if (lane == 0) wmax[wave] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) most = max(most, wmax[w]);
        const bool bad = most >= kInfBits;
        scale = scale_of(most);
        const float inv = 1.0f / scale;
        int32_t sum = 0;
#pragma unroll
        for (int i = 0; i < kHold; ++i) {
            const int k = (i * NW * 64 + tid) * 8;
            if (k >= K) continue;
            uint32_t b[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = code_bits(xr[i][e], inv);
            uint2 v = make_uint2(pack_codes(b[0], b[1], b[2], b[3]),
                                 pack_codes(b[4], b[5], b[6], b[7]));
            if (bad) v = make_uint2(0, 0);
            *reinterpret_cast<uint2*>(smem + k) = v;
            sum = __builtin_amdgcn_sdot4((int)v.x, 0x01010101, sum, false);
            sum = __builtin_amdgcn_sdot4((int)v.y, 0x01010101, sum, false);
        }
        if (bad) scale = __builtin_nanf("");
        if (p.w_zp) {
            sum = (int32_t)wave_sum(sum);
            if (lane == 0) wsum[wave] = sum;
        }
    }
    __syncthreads();
    if (FUSED && p.w_zp) {
#pragma unroll
        for (int w = 0; w < NW; ++w) rs += wsum[w];
    }

    // |sum| <= K 2^14 <= 2^30 (4-bit weights as 16 w): exact
    int32_t acc = 0;
    for (int s = s_begin; s < s_end; s += kSteps) {
        if (s != s_begin) load(s);
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
            const int off = ((s + u) * kLanes + j) * 16;
            if constexpr (WBITS == 8) {
                const v4i x = *reinterpret_cast<const v4i*>(smem + (off < wrow ? off : 0));
#pragma unroll
                for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_sdot4(wv[u][q], x[q], acc, false);
            } else {
                const int kk = off < wrow ? 2 * off : 0;
                const v4i w0 = unpack_int4_x16((uint32_t)wv[u][0], (uint32_t)wv[u][1]);
                const v4i w1 = unpack_int4_x16((uint32_t)wv[u][2], (uint32_t)wv[u][3]);
                const v4i x0 = *reinterpret_cast<const v4i*>(smem + kk);
                const v4i x1 = *reinterpret_cast<const v4i*>(smem + kk + 16);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_sdot4(w0[q], x0[q], acc, false);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_sdot4(w1[q], x1[q], acc, false);
            }
        }
    }
    acc += __shfl_xor(acc, 1);
    acc += __shfl_xor(acc, 2);
    acc += __shfl_xor(acc, 4);
    if (j == 0) red[wave * kChans + c] = acc;
    __syncthreads();
    if (!epi || n0 + lane >= p.N) return;
    int32_t sum = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += red[w * kChans + lane];
    if constexpr (WBITS == 4) sum >>= 4;  // exact: a multiple of 16
    sum -= zw * rs;
    store_out(a.t, n0 + lane, token_output(sum, ws, scale, bias));
}

template <int NW>
constexpr int64_t one_token_lds(int64_t K)
{
    return (K + 15) / 16 * 16 + NW * (kChans + 2) * 4;
}

template <int WBITS, int XTYPE, int NW>
hipError_t launch_one(const OneArgs& a, hipStream_t s)
{
    // more than 64 KiB of dynamic LDS has to be opted into
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&one_token_kernel<WBITS, XTYPE, NW>),
                            hipFuncAttributeMaxDynamicSharedMemorySize,
                            (int)one_token_lds<NW>(MQ_MAX_K));
    if (attr != hipSuccess) return attr;
    one_token_kernel<WBITS, XTYPE, NW><<<(unsigned)((a.p.N + kChans - 1) / kChans), NW * 64,
                                         (size_t)one_token_lds<NW>(a.p.K), s>>>(a);
    return hipGetLastError();
}

// waves: enough that one round of loads covers each wave's share of a row, at
// most eight
int one_token_waves(const QLinearArgs& p)
{
    const int64_t wrow = p.w_bits == 8 ? p.K : p.K / 2;
    const int64_t steps = (wrow + kLanes * 16 - 1) / (kLanes * 16);
    int nw = 1;
    while (nw < 8 && nw * kSteps < steps) nw *= 2;
    return nw;
}

template <int WBITS, int XTYPE>
hipError_t launch_one_nw(const OneArgs& a, hipStream_t s)
{
    switch (one_token_waves(a.p)) {
    case 8: return launch_one<WBITS, XTYPE, 8>(a, s);
    case 4: return launch_one<WBITS, XTYPE, 4>(a, s);
    case 2: return launch_one<WBITS, XTYPE, 2>(a, s);
    default: return launch_one<WBITS, XTYPE, 1>(a, s);
    }
}

template <int XTYPE>
hipError_t launch_one_w(const OneArgs& a, hipStream_t s)
{
    return a.p.w_bits == 8 ? launch_one_nw<8, XTYPE>(a, s) : launch_one_nw<4, XTYPE>(a, s);
}

// ---------------------------------------------------------------------------
// 2 to 16 tokens: R channels per work-group (8, or tiles of 16), its waves split K; a
// lane streams 16 weights of one channel of each tile per step and the MFMA multiplies
// them with the tokens (zeros past the last), whose codes a wave reads once for all
// tiles.  A load takes half a line of each row: read past the caches the lines came
// twice (16 x 2048 -> 8192: 7.3 us, 6.4 through them).  What bounds it: reads, 2.7 TB/s of
// weights at that size, whose waves have one round of loads; where there are more, a way
// to memory for each, since a round is asked for behind the products of the one before
// (16 x 5632 -> 2048 of 4 bits, three rounds: 7.1 us; 16384 -> 2048 of 8 bits, four: 14.4).
template <int WBITS, int NWAVES, int R>
__global__ __launch_bounds__(NWAVES * 64) void few_tokens_kernel(QLinearArgs p, TokenArgs t)
{
    constexpr int RT = R > 16 ? R / 16 : 1;  // tiles
    constexpr int U = 8;                     // 64-deep steps per round of loads
    static_assert(NWAVES >= RT, "a wave per tile in the end");
    __shared__ v4i red[NWAVES][RT][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, kg = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * R;
    const int K = (int)p.K;
    const int wrow = WBITS == 8 ? K : K / 2;
    const int rows = (int)(p.N - n0 < R ? p.N - n0 : R);
    // loads past a row's, the channels' or the tokens' end return zeros
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(static_cast<const int8_t*>(p.w) + n0 * wrow), (short)0, rows * wrow, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra =
        __builtin_amdgcn_make_buffer_rsrc((void*)p.a, (short)0, (int)(p.M * K), 0x00020000);
    const int m = r16 < (int)p.M ? r16 : (int)p.M - 1;
    const uint32_t a_dead = r16 < (int)p.M ? 0u : kOOB;

    // wave q ends tile q: token r16, channels c0 + {0..3}
    const int64_t c0 = n0 + 16 * wave + 4 * kg;
    float ws[4], bias[4], ts = 0.0f;
    int32_t zw[4], rs = 0;
    if (wave < RT) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            int64_t n = c0 + r;
            if (n >= p.N) n = p.N - 1;
            ws[r] = p.w_scale[n];
            bias[r] = p.bias ? p.bias[n] : -0.0f;
            zw[r] = p.w_zp ? p.w_zp[n] : 0;
        }
        ts = t.scale[m];
        if (p.w_zp) rs = p.a_rowsum[m];
    }
    const int steps = (K + 63) / 64;
    const int s_begin = steps * wave / NWAVES, s_end = steps * (wave + 1) / NWAVES;
    v4i wv[U][RT], av[U];
    auto load = [&](int s) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s + u) * 64 + kg * 16;
            const uint32_t dead = (uint32_t)((s + u >= s_end) | (k >= K)) << 31;
#pragma unroll
            for (int q = 0; q < RT; ++q) {
                const int row = 16 * q + r16;
                if constexpr (WBITS == 8) {
                    wv[u][q] = __builtin_amdgcn_raw_buffer_load_b128(
                        rw, (uint32_t)(row * K + k) | dead, 0, 0);
                } else {
                    typedef unsigned v2u __attribute__((ext_vector_type(2)));
                    const v2u pk = __builtin_amdgcn_raw_buffer_load_b64(
                        rw, (uint32_t)(row * wrow + k / 2) | dead, 0, 0);
                    wv[u][q] = v4i{(int)pk[0], (int)pk[1], 0, 0};
                }
            }
            av[u] = __builtin_amdgcn_raw_buffer_load_b128(
                ra, (uint32_t)(r16 * K + k) | dead | a_dead, 0, 0);
        }
    };
    v4i acc[RT];
#pragma unroll
    for (int q = 0; q < RT; ++q) acc[q] = v4i{0, 0, 0, 0};
    for (int s = s_begin; s < s_end; s += U) {
        load(s);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < RT; ++q) {
                v4i w = wv[u][q];
                if constexpr (WBITS == 4) w = unpack_int4_x16((uint32_t)w[0], (uint32_t)w[1]);
                acc[q] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w, av[u], acc[q], 0, 0, 0);
            }
    }
    v4i sum = acc[0];
    if constexpr (NWAVES > 1) {
#pragma unroll
        for (int q = 0; q < RT; ++q) red[wave][q][lane] = acc[q];
        __syncthreads();
        if (wave >= RT) return;
        sum = red[0][wave][lane];
#pragma unroll
        for (int w = 1; w < NWAVES; ++w) sum += red[w][wave][lane];
    }
    if (r16 >= (int)p.M || 4 * kg >= R) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t n = c0 + r;
        if (n >= p.N) break;
        int32_t c = sum[r];
        if constexpr (WBITS == 4) c >>= 4;  // exact: a multiple of 16
        c -= zw[r] * rs;
        store_out(t, r16 * p.N + n, token_output(c, ws[r], ts, bias[r]));
    }
}

template <int WBITS, int R>
hipError_t launch_few_r(const QLinearArgs& p, const TokenArgs& t, hipStream_t s)
{
    const int64_t blocks = (p.N + R - 1) / R, steps = (p.K + 63) / 64;
    // waves: a round of loads each, up to four (at least four where there are few
    // work-groups); eight from four rounds on (16 x 5632 -> 2048 of 4 bits: 6.8 us with
    // four, 7.3 with eight; 16384 -> 2048 of 8 bits: 18.4 and 15.3)
    int nw = R > 16 ? R / 16 : 1;
    while (nw < 4 && (nw * 8 < steps || (blocks < 2048 && nw < steps))) nw *= 2;
    if (nw == 4 && nw * 32 < steps) nw = 8;
    const unsigned b = (unsigned)blocks;
    switch (nw) {
    case 8: few_tokens_kernel<WBITS, 8, R><<<b, 512, 0, s>>>(p, t); break;
    case 4: few_tokens_kernel<WBITS, 4, R><<<b, 256, 0, s>>>(p, t); break;
    case 2: few_tokens_kernel<WBITS, 2, R><<<b, 128, 0, s>>>(p, t); break;
    default:
        if constexpr (R <= 16) few_tokens_kernel<WBITS, 1, R><<<b, 64, 0, s>>>(p, t);
    }
    return hipGetLastError();
}

template <int WBITS>
hipError_t launch_few(const QLinearArgs& p, const TokenArgs& t, hipStream_t s)
{
    // enough work-groups to stream, then fewer reads of the tokens' codes: with 8, 16 and
    // 32 channels per work-group 16 x 2048 -> 2048 takes 4.1, 4.3 and 5.2 us, -> 4096 6.0,
    // 4.8 and 5.8, -> 8192 9.7, 7.3 and 6.2
    if (p.N < 4096) return launch_few_r<WBITS, 8>(p, t, s);
    return p.N < 8192 ? launch_few_r<WBITS, 16>(p, t, s) : launch_few_r<WBITS, 32>(p, t, s);
}

// ---------------------------------------------------------------------------
// Any shape and alignment: one thread per output.
template <int WBITS>
__global__ __launch_bounds__(256) void any_tokens_kernel(QLinearArgs p, TokenArgs t)
{
    const int64_t total = p.M * p.N, stride = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += stride) {
        const int64_t m = i / p.N, n = i - m * p.N;
        const int8_t* x = p.a + m * p.K;
        int32_t acc = 0;
        if constexpr (WBITS == 8) {
            const int8_t* w = static_cast<const int8_t*>(p.w) + n * p.K;
            for (int64_t k = 0; k < p.K; ++k) acc += (int32_t)x[k] * (int32_t)w[k];
        } else {
            const uint8_t* w = static_cast<const uint8_t*>(p.w) + n * (p.K / 2);
            for (int64_t k = 0; k < p.K / 2; ++k) {
                const int32_t b = w[k];
                acc += (int32_t)x[2 * k] * ((int32_t)((uint32_t)b << 28) >> 28) +
                       (int32_t)x[2 * k + 1] * ((int32_t)((uint32_t)b << 24) >> 28);
            }
        }
        if (p.w_zp) acc -= p.w_zp[n] * p.a_rowsum[m];
        store_out(t, i, token_output(acc, p.w_scale[n], t.scale[m], p.bias ? p.bias[n] : -0.0f));
    }
}

hipError_t launch_any(const QLinearArgs& p, const TokenArgs& t, hipStream_t s)
{
    const int64_t blocks = (p.M * p.N + 255) / 256;
    const unsigned b = (unsigned)(blocks > 256 * 64 ? 256 * 64 : blocks);
    if (p.w_bits == 8) any_tokens_kernel<8><<<b, 256, 0, s>>>(p, t);
    else any_tokens_kernel<4><<<b, 256, 0, s>>>(p, t);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// More than 16 tokens.
template <class C, bool ASYM>
__global__ __launch_bounds__(C::THREADS, C::OCC) void token_tiles_kernel(QLinearArgs p, TokenArgs t,
                                                                         int tiles_n, int tiles_m,
                                                                         int splits,
                                                                         int kt_per_split)
{
    prefill_body<C, ASYM, false, false, true>(p, nullptr, tiles_n, tiles_m, splits, kt_per_split,
                                              &t);
}

template <class C, bool ASYM>
hipError_t launch_tiles(const QLinearArgs& p, const TokenArgs& t, int splits, hipStream_t s)
{
    const int64_t tiles_n = (p.N + C::TN - 1) / C::TN, tiles_m = (p.M + C::TM - 1) / C::TM;
    const int64_t total = tiles_n * tiles_m, kt = (p.K + C::BK - 1) / C::BK;
    const int64_t per = (kt + splits - 1) / splits;
    splits = (int)((kt + per - 1) / per);  // every slice non-empty
    if (total * splits > 0x7FFFFFFF) return hipErrorInvalidValue;
    constexpr int lds = C::LDS_ASYM;  // (the token scales lie where 16-bit codes' row terms do)
    static const hipError_t attr =
        hipFuncSetAttribute(reinterpret_cast<const void*>(&token_tiles_kernel<C, ASYM>),
                            hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    token_tiles_kernel<C, ASYM><<<(unsigned)(total * splits), C::THREADS, lds, s>>>(
        p, t, (int)tiles_n, (int)tiles_m, splits, (int)per);
    return hipGetLastError();
}

template <int WB, bool ASYM>
hipError_t launch_tiles_a(const QLinearArgs& p, const TokenArgs& t, hipStream_t s)
{
    Choice ch = choose(p, p.ws != nullptr);
    if (ch.splits > 1 && workspace_for(p, ch) > p.ws_bytes) ch = choose(p, false);
    switch (ch.tile) {
    case kTile256x128: return launch_tiles<T256x128<WB, 16>, ASYM>(p, t, ch.splits, s);
    case kTile192x256: return launch_tiles<T192x256<WB, 16>, ASYM>(p, t, ch.splits, s);
    case kTile64x64: return launch_tiles<T64x64<WB, 16>, ASYM>(p, t, ch.splits, s);
    case kTile256x256W8: return launch_tiles<T256x256W8<WB, 16>, ASYM>(p, t, ch.splits, s);
    case kTile64x128: return launch_tiles<T64x128<WB, 16>, ASYM>(p, t, ch.splits, s);
    default: return launch_tiles<T128x128<WB, 16>, ASYM>(p, t, ch.splits, s);
    }
}

template <int WB>
hipError_t launch_tiles_w(const QLinearArgs& p, const TokenArgs& t, hipStream_t s)
{
    return p.w_zp ? launch_tiles_a<WB, true>(p, t, s) : launch_tiles_a<WB, false>(p, t, s);
}

// Whole 16-byte chunks of aligned rows (8-byte ones of packed 4-bit weights for
// the few tokens' kernel, whose K is a multiple of 16).
bool rows_ok(const QLinearArgs& p, int chunk4)
{
    return p.K % (p.w_bits == 8 ? 16 : 2 * chunk4) == 0 && (uintptr_t)p.a % 16 == 0 &&
           (uintptr_t)p.w % (p.w_bits == 8 ? 16 : chunk4) == 0;
}

// (byte offsets inside a 256-row tile fit 31 bits)
bool tiles_ok(const QLinearArgs& p, int32_t y_type)
{
    return rows_ok(p, 16) && 256 * p.N * type_bytes(y_type) < kOOB && 256 * p.K < kOOB;
}

}  // namespace

bool one_token_fused(const QLinearArgs& p, const void* x)
{
    // Every work-group quantizes the token once more, which costs a launch's time at
    // about so many elements in all: in one launch and two (weights from memory, 8 and
    // 4 bits), 2048 -> 5632 4.4 and 6.1, 3.8 and 5.4 us; 2048 -> 256000 81 and 85, 42
    // and 46; 5632 -> 131072 115 and 117, 76 and 75; 5632 -> 256000 225 and 223, 148 and
    // 135.
    constexpr int64_t kMost = (int64_t)1 << 26;
    return p.M == 1 && rows_ok(p, 16) && (uintptr_t)x % 16 == 0 &&
           (p.N + kChans - 1) / kChans * p.K <= kMost &&
           p.K <= (int64_t)one_token_waves(p) * 64 * 8 * kHold;
}

bool few_tokens_in_tiles(const QLinearArgs& p, int32_t y_type)
{
    // The tiles read the weights in whole lines, and 16 tokens cost them what 2 do: 2, 6
    // and 16 tokens of 2048 -> 16384 take the few tokens' kernel 9.0, 9.3 and 10.5 us, the
    // tiles 8.9; -> 131072 62, 59 and 73, the tiles 55 to 61 (4 bits 41, 44, 57 and 33).
    return p.M > 1 && p.N >= 16384 && tiles_ok(p, y_type);
}

hipError_t launch_linear_one_token(const QLinearArgs& p, const TokenArgs& t, const void* x,
                                   int32_t type, hipStream_t s)
{
    const OneArgs a{p, t, x};
    if (type == MQ_F32) return launch_one_w<MQ_F32>(a, s);
    return type == MQ_BF16 ? launch_one_w<MQ_BF16>(a, s) : launch_one_w<MQ_F16>(a, s);
}

hipError_t launch_qlinear_tokens(const QLinearArgs& p, const TokenArgs& t, int32_t path,
                                 hipStream_t s)
{
    if (path == MQ_PATH_DECODE) {
        if (p.M == 1 && rows_ok(p, 16)) return launch_one_w<-1>(OneArgs{p, t, nullptr}, s);
        if (rows_ok(p, 8))
            return p.w_bits == 8 ? launch_few<8>(p, t, s) : launch_few<4>(p, t, s);
    }
    if (path == MQ_PATH_PREFILL && tiles_ok(p, t.type))
        return p.w_bits == 8 ? launch_tiles_w<8>(p, t, s) : launch_tiles_w<4>(p, t, s);
    return launch_any(p, t, s);
}

}  // namespace mq
