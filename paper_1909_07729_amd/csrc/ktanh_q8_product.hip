// libktanh: products of rows in 8-bit integers with weights in 8-bit integers, scaled by row and by output channel.
//
//   out[t][o] = (float(sum over i of x[t][i] * w[o][i]) * x_scale[t]) * w_scale[o] + bias[o]
//
// The sums are exact (32-bit integers); the scaling is Float32, one rounding per operation.
#include <type_traits>

#include "ktanh_q8.h"
#include "ktanh_q8_device.h"

using namespace ktanh_device;
using namespace ktanh_q8;

namespace {

// ------------------------------------------------------------------------------------ tiles
// Products of many rows.  A block of four wavefronts has TO output channels and TT rows, each wavefront a quarter of it (two by two, or four along the
// channels where the rows are 32).  Tiles of 128 integers of the inner dimension come into LDS by direct loads, into a ring of PLACES; operands are read a step
// of 32 integers ahead of the products that take them, and the place of a tile is filled again between its last products, when it has been read.
//
// What bounds it: with many rows the matrix cores and the clock under them (8192 x 16384 x 4096 477 us, 2300 TOP/s, 58 % of the cycles at 1.75 GHz; its
// operands pass LDS, 1 KB for 64 products at 256 by 256, where 128 by 128 needs twice that); with few rows the weights' way from memory (64 x 4096 x 16384 13.4 us from
// the last-level cache, 5.2 TB/s, 19 from memory; 24 x 2048 x 50000 21 us, 5.0 TB/s).
//
// Rows of a tile are 128 bytes, half of the width of LDS.  Chunks of 16 bytes change places with bits 1 to 3 of their row's number, so that sixteen
// neighbouring rows at one chunk, which are read at once, lie in different banks.
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
constexpr unsigned kDeep = 128;     // integers of a tile

// 16 bytes of each lane from `base` + its offset to LDS, at `to` + 16 * lane, with no register between.  As an instruction, because the compiler
// would wait for all such loads before any read of LDS that it cannot tell apart from them; wait_for_tiles counts them instead.  (Nothing else in these
// kernels uses M0.)
__device__ __forceinline__ void load_direct(const int8_t *base, unsigned offset, char *to)
{
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)to;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(__builtin_amdgcn_readfirstlane(at)), "v"(offset), "s"(base) : "memory");
}
// All but the last LOADS of this wavefront's loads have arrived, and its reads of LDS are done.
template <unsigned LOADS>
__device__ __forceinline__ void wait_for_tiles()
{
    static_assert(LOADS < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((LOADS & 15) | 7 << 4 | (LOADS >> 4) << 14);
}

// R rows of an operand, of which `there` are inside (the rest is read as the last), brought to LDS by the block.
template <unsigned R>
struct Side {
    const int8_t *base;         // the tile's first row
    unsigned offset[R / 32];    // of this lane's chunks
    static constexpr unsigned kLoads = R / 32;

    // The chunk that a lane brings to place lane % 8 of row 8 i + lane / 8.
    __device__ __forceinline__ static unsigned chunk_of(unsigned i) { return threadIdx.x % 8 ^ (threadIdx.x / 64 * (R / 8) + 4 * i + threadIdx.x % 64 / 16) % 8; }

    __device__ __forceinline__ Side(const int8_t *rows, unsigned long long row, unsigned first, unsigned last)
    {
        const unsigned lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        base = rows + first * row;
#pragma unroll
        for (unsigned i = 0; i < kLoads; ++i) {
            const unsigned at = wave * (R / 4) + i * 8 + lane / 8, most = last - first;
            offset[i] = (at < most ? at : most) * (unsigned)row + chunk_of(i) * 16;
        }
    }
    __device__ __forceinline__ void load(unsigned i, unsigned k, char *tile) const
    {
        load_direct(base + k, offset[i], tile + (__builtin_amdgcn_readfirstlane(threadIdx.x / 64) * (R / 4) + i * 8) * kDeep);
    }
    // The end of the rows, fewer than kDeep integers, zeros behind them: asked for before the tiles, put into place behind them.
    i32x4 end[kLoads];
    __device__ __forceinline__ void ask_end(unsigned k, unsigned inner)
    {
#pragma unroll
        for (unsigned i = 0; i < kLoads; ++i) end[i] = ask16(base + k + offset[i], (int)(inner - k) - (int)(chunk_of(i) * 16), inner);
    }
    __device__ __forceinline__ void take_end(unsigned k, unsigned inner, char *tile)
    {
        const unsigned lane = threadIdx.x % 64;
#pragma unroll
        for (unsigned i = 0; i < kLoads; ++i) {
            asm volatile("" : "+v"(end[i]));
            *reinterpret_cast<i32x4 *>(tile + (threadIdx.x / 64 * (R / 4) + i * 8) * kDeep + lane * 16) =
                take16(end[i], base + k + offset[i], (int)(inner - k) - (int)(chunk_of(i) * 16), inner);
        }
    }
};

// Which tile a block takes.  Blocks go to the eight XCDs in turn, each with an L2 of its own: each XCD gets a run of tiles, and a run goes through four tiles
// of rows at a time, so that the blocks that an XCD works on at once share rows and channels.
struct Corner {
    unsigned over, across;
};
__device__ __forceinline__ Corner corner_of(unsigned block, unsigned over, unsigned across)
{
    constexpr unsigned kRows = 4;
    const unsigned each = over * across / 8, id = block < 8 * each ? block % 8 * each + block / 8 : block;
    const unsigned group = id / (kRows * over), in = id % (kRows * over), rows = across - group * kRows < kRows ? across - group * kRows : kRows;
    return Corner{in / rows, group * kRows + in % rows};
}

template <unsigned TO, unsigned TT, unsigned PLACES, Out OUT>
__global__ __launch_bounds__(256, PLACES * (TO + TT) * kDeep > 81920 ? 1 : 2) void q8_tile_kernel(Operands a, unsigned over, unsigned across, unsigned parts)
{
    constexpr unsigned WT = TT < 64 ? 1 : 2, WO = 4 / WT;       // wavefronts side by side along the rows, and along the channels
    constexpr unsigned OI = TO / WO / 32, TI = TT / WT / 32, kPlace = (TO + TT) * kDeep;
    __shared__ __align__(16) char lds[PLACES * kPlace];
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned part = blockIdx.x / (over * across);
    const Corner at = corner_of(blockIdx.x - part * (over * across), over, across);
    const unsigned o0 = at.over * TO, t0 = at.across * TT;
    Side<TO> w(a.w, a.w_row, o0, a.outer - 1);
    Side<TT> x(a.x, a.x_row, t0, a.rows - 1);
    constexpr unsigned kLoads = w.kLoads + x.kLoads;
    auto load = [&](unsigned n, unsigned k, char *place) {
        if (n < w.kLoads) w.load(n, k, place);
        else x.load(n - w.kLoads, k, place + TO * kDeep);
    };
    i32x16 sum[OI][TI];
#pragma unroll
    for (unsigned i = 0; i < OI; ++i)
#pragma unroll
        for (unsigned j = 0; j < TI; ++j) sum[i][j] = i32x16{0};
    // operands of 32 integers: a lane has 16 of one row
    const unsigned w_at = (wave / WT * (TO / WO) + lane % 32) * kDeep, x_at = TO * kDeep + (wave % WT * (TT / WT) + lane % 32) * kDeep;
    i32x4 wf[2][OI], xf[2][TI];
    auto read = [&](const char *place, unsigned step) {
        const unsigned chunk = ((2 * step + lane / 32) ^ lane / 2 % 8) * 16;
#pragma unroll
        for (unsigned i = 0; i < OI; ++i) wf[step % 2][i] = *reinterpret_cast<const i32x4 *>(place + w_at + chunk + i * 32 * kDeep);
#pragma unroll
        for (unsigned j = 0; j < TI; ++j) xf[step % 2][j] = *reinterpret_cast<const i32x4 *>(place + x_at + chunk + j * 32 * kDeep);
    };
    auto multiply = [&](unsigned step, auto between) {
#pragma unroll
        for (unsigned i = 0; i < OI; ++i)
#pragma unroll
            for (unsigned j = 0; j < TI; ++j) {
                sum[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[step % 2][i], xf[step % 2][j], sum[i][j], 0, 0, 0);
                between(i * TI + j);
            }
    };
    auto nothing = [](unsigned) {};
    // this block's tiles of the inner dimension; the last part has what is left of a tile as well
    const unsigned all = a.inner / kDeep, from = (unsigned)((unsigned long long)all * part / parts),
                   tiles = (unsigned)((unsigned long long)all * (part + 1) / parts) - from;
    // Without a branch: past the last tiles the last one is asked for again, into a place that nobody reads, and what is read ahead is not used.
    auto tile_at = [&](unsigned tile) { return (from + (tile < tiles ? tile : tiles - 1)) * kDeep; };
    auto step = [&](unsigned tile, char *here, const char *next) {
#pragma unroll
        for (unsigned s = 0; s < 3; ++s) {
            read(here, s + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(s, nothing);
            __builtin_amdgcn_sched_barrier(0);
        }
        // the next tile is complete, and this one has been read by all
        wait_for_tiles<kLoads * (PLACES - 2)>();
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        read(next, 0);
        __builtin_amdgcn_sched_barrier(0);
        const unsigned k = tile_at(tile + PLACES);
        multiply(3, [&](unsigned n) {
            constexpr unsigned kEach = (kLoads + OI * TI - 1) / (OI * TI);
#pragma unroll
            for (unsigned e = 0; e < kEach; ++e)
                if (n * kEach + e < kLoads) load(n * kEach + e, k, here);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    const bool ragged = part + 1 == parts && a.inner % kDeep != 0;
    const unsigned o1 = o0 + wave / WT * (TO / WO), t1 = t0 + wave % WT * (TT / WT);
    const bool biased = a.bias != nullptr;
    f32x4 channel[OI][4], bias[OI][4];
    float row[TI];
    auto ask_scales = [&] {
        if constexpr (OUT == SUMS) return;
#pragma unroll
        for (unsigned i = 0; i < OI; ++i)
#pragma unroll
            for (unsigned q = 0; q < 4; ++q) {
                const unsigned o = o1 + i * 32 + q * 8 + lane / 32 * 4;
                channel[i][q] = four_of(a.w_scale, o, a.outer);
                bias[i][q] = biased ? four_of(a.bias, o, a.outer) : f32x4{0, 0, 0, 0};
            }
    };
    auto ask_row = [&](unsigned j) {
        const unsigned t = t1 + j * 32 + lane % 32;
        if constexpr (OUT != SUMS) row[j] = a.x_scale[t < a.rows ? t : a.rows - 1];
    };
    // what the small tiles need at their end is asked for first (777 x 1001 x 2003 10.5 us, 11.5 with all of it behind the tiles); the large ones have no registers for it
    constexpr bool kEarly = TO * TT <= 128 * 128;
    if constexpr (kEarly) {
        ask_scales();
#pragma unroll
        for (unsigned j = 0; j < TI; ++j) ask_row(j);
    }
    if (kEarly && ragged) {
        w.ask_end(all * kDeep, a.inner);
        x.ask_end(all * kDeep, a.inner);
    }
    if (tiles != 0) {
#pragma unroll
        for (unsigned p = 0; p < PLACES; ++p)
#pragma unroll
            for (unsigned n = 0; n < kLoads; ++n) load(n, tile_at(p), lds + p * kPlace);
        wait_for_tiles<kLoads * (PLACES - 1)>();
        __syncthreads();
        read(lds, 0);
        unsigned here = 0;
        for (unsigned tile = 0; tile < tiles; ++tile) {
            const unsigned next = here + 1 < PLACES ? here + 1 : 0;
            step(tile, lds + here * kPlace, lds + next * kPlace);
            here = next;
        }
        wait_for_tiles<0>();
    }
    char *const first = lds;
    if (ragged) {
        if constexpr (!kEarly) {
            w.ask_end(all * kDeep, a.inner);
            x.ask_end(all * kDeep, a.inner);
        }
        __syncthreads();
        w.take_end(all * kDeep, a.inner, first);
        x.take_end(all * kDeep, a.inner, first + TO * kDeep);
        __syncthreads();
#pragma unroll
        for (unsigned s = 0; s < 4; ++s) {
            read(first, s);
            multiply(s, nothing);
        }
    }
    // A lane has, of 32 channels and 32 rows, four times 4 neighbouring channels of one row.  The results of 32 rows go through a wavefront's own
    // place in LDS, and leave by whole rows of its channels: straight from the registers each store would touch 32 rows, 16 bytes of each.
    __syncthreads();
    constexpr unsigned kSize = OUT == BF16 ? 2 : 4, kRow = TO / WO * kSize, kPitch = kRow + 16, kChunks = kRow / 16;
    static_assert(4 * 32 * kPitch <= PLACES * kPlace, "four wavefronts' results");
    char *const mine = lds + wave * 32 * kPitch;
    if constexpr (OUT == SUMS) a.out = static_cast<float *>(a.out) + (unsigned long long)part * a.rows * a.outer;
    if constexpr (!kEarly) ask_scales();
#pragma unroll
    for (unsigned j = 0; j < TI; ++j) {
        if constexpr (!kEarly) ask_row(j);
#pragma unroll
        for (unsigned i = 0; i < OI; ++i)
#pragma unroll
            for (unsigned q = 0; q < 4; ++q) {
                const i32x4 four = {sum[i][j][4 * q], sum[i][j][4 * q + 1], sum[i][j][4 * q + 2], sum[i][j][4 * q + 3]};
                f32x4 y;
                if constexpr (OUT == SUMS) y = __builtin_bit_cast(f32x4, four);
                else y = scaled(four, row[j], channel[i][q], bias[i][q], biased);
                put_four<OUT>(mine + lane % 32 * kPitch + (i * 32 + q * 8 + lane / 32 * 4) * kSize, y);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
#pragma unroll
        for (unsigned n = 0; n < 32 * kChunks / 64; ++n) {
            const unsigned at = (n * 64 + lane) / kChunks, chunk = (n * 64 + lane) % kChunks;
            store_chunk<OUT>(a, t1 + j * 32 + at, o1 + chunk * Result<OUT>::kEach, *reinterpret_cast<const u32x4 *>(mine + at * kPitch + chunk * 16));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
    }
}

// ------------------------------------------------------------------------------------ a shared inner dimension
// A block has OT output channels and TT rows, and its W wavefronts share the inner dimension in steps of 64 integers: wavefront s takes the steps
// s, s + W, ..., so that the block reads whole cache lines.  Operands go from memory to the matrix cores' registers; the wavefronts' sums
// meet in LDS.  Bound by latency and the weights' way from memory: 1 x 4096 x 4096 takes 5.5 us from the last-level cache (3.1 TB/s, launch included), 64 x 1024 x 1024 3.4.
template <unsigned OT, unsigned TT, unsigned W, Out OUT, bool ALIGNED>
__global__ __launch_bounds__(64 * W) void q8_shared_inner_kernel(Operands a)
{
    constexpr unsigned OI = OT / 16, TI = TT / 16;
    __shared__ int part[W][TT][OT + 4];
    const unsigned lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned o0 = blockIdx.x * OT, t0 = blockIdx.y * TT;
    // rows past the last are read as the last, and not stored
    const int8_t *w[OI], *x[TI];
    const unsigned k = lane / 16 * 16;
#pragma unroll
    for (unsigned i = 0; i < OI; ++i) {
        const unsigned o = o0 + 16 * i + lane % 16;
        w[i] = a.w + (o < a.outer ? o : a.outer - 1) * a.w_row + k;
    }
#pragma unroll
    for (unsigned i = 0; i < TI; ++i) {
        const unsigned t = t0 + 16 * i + lane % 16;
        x[i] = a.x + (t < a.rows ? t : a.rows - 1) * a.x_row + k;
    }
    i32x4 sum[OI][TI];
#pragma unroll
    for (unsigned i = 0; i < OI; ++i)
#pragma unroll
        for (unsigned j = 0; j < TI; ++j) sum[i][j] = i32x4{0, 0, 0, 0};
    auto multiply = [&](const i32x4 (&wf)[OI], const i32x4 (&xf)[TI]) {
#pragma unroll
        for (unsigned i = 0; i < OI; ++i)
#pragma unroll
            for (unsigned j = 0; j < TI; ++j) sum[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[i], xf[j], sum[i][j], 0, 0, 0);
    };
    // Whole groups of U steps, the next group's operands on their way during the products of one.
    constexpr unsigned U = OI + TI > 4 ? 2 : OI + TI > 2 ? 4 : 8;
    const unsigned whole = a.inner / 64, mine = whole > wave ? (whole - wave + W - 1) / W : 0, groups = mine / U;
    i32x4 wf[2][U][OI], xf[2][U][TI];
    auto load = [&](unsigned to, unsigned group) {
        if (group >= groups) return;
        const unsigned at = (wave + group * U * W) * 64;
#pragma unroll
        for (unsigned u = 0; u < U; ++u) {
#pragma unroll
            for (unsigned i = 0; i < OI; ++i) wf[to][u][i] = load16<ALIGNED>(w[i] + at + u * W * 64);
#pragma unroll
            for (unsigned i = 0; i < TI; ++i) xf[to][u][i] = load16<ALIGNED>(x[i] + at + u * W * 64);
        }
    };
    load(0, 0);
    for (unsigned g = 0; g < groups; g += 2) {
        load(1, g + 1);
#pragma unroll
        for (unsigned u = 0; u < U; ++u) multiply(wf[0][u], xf[0][u]);
        load(0, g + 2);
        if (g + 1 < groups) {
#pragma unroll
            for (unsigned u = 0; u < U; ++u) multiply(wf[1][u], xf[1][u]);
        }
    }
    unsigned s = wave + groups * U * W;
    for (; s * 64 < a.inner; s += W) {
        const int there = (int)a.inner - (int)(s * 64 + k);
        i32x4 w1[OI], x1[TI];
#pragma unroll
        for (unsigned i = 0; i < OI; ++i) w1[i] = load16(w[i] + s * 64, there, a.inner);
#pragma unroll
        for (unsigned i = 0; i < TI; ++i) x1[i] = load16(x[i] + s * 64, there, a.inner);
        multiply(w1, x1);
    }
    // a lane has 4 neighbouring channels of a row
#pragma unroll
    for (unsigned i = 0; i < OI; ++i)
#pragma unroll
        for (unsigned j = 0; j < TI; ++j)
            *reinterpret_cast<i32x4 *>(&part[wave][16 * j + lane % 16][16 * i + lane / 16 * 4]) = sum[i][j];
    __syncthreads();
    store_joined<OT, TT, W, OUT>(a, o0, t0, part);
}

// ------------------------------------------------------------------------------------ parts joined
// The sums of the parts of the inner dimension added up, scaled and stored; a chunk of 16 bytes to a lane.  Bound by memory and its launch: 4 parts of
// 512 x 1024 take 3 us.
template <Out OUT>
__global__ __launch_bounds__(256) void q8_join_kernel(Operands a, const int *sums, unsigned parts)
{
    constexpr unsigned E = Result<OUT>::kEach;
    const unsigned across = (a.outer + E - 1) / E;
    const unsigned long long id = blockIdx.x * 256ull + threadIdx.x;
    if (id >= (unsigned long long)across * a.rows) return;
    const unsigned t = (unsigned)(id / across), o = (unsigned)(id % across) * E;
    const unsigned long long each = (unsigned long long)a.rows * a.outer;
    typedef i32x4 anywhere __attribute__((aligned(4)));
    const float row = a.x_scale[t];
    const bool biased = a.bias != nullptr;
    u32x4 out;
#pragma unroll
    for (unsigned h = 0; h < E / 4; ++h) {
        const unsigned c = o + 4 * h;
        if (c >= a.outer) break;
        i32x4 v = {0, 0, 0, 0};
        for (unsigned p = 0; p < parts; ++p) {
            const int *from = sums + p * each + t * (unsigned long long)a.outer + c;
            if (c + 4 <= a.outer) {
                v += *reinterpret_cast<const anywhere *>(from);
            } else {
                for (unsigned i = 0; i < 3; ++i)
                    if (c + i < a.outer) v[i] += from[i];
            }
        }
        put_four<OUT>(reinterpret_cast<char *>(&out) + 8 * h,
                      scaled(v, row, four_of(a.w_scale, c, a.outer), biased ? four_of(a.bias, c, a.outer) : f32x4{0, 0, 0, 0}, biased));
    }
    store_chunk<OUT>(a, t, o, out);
}

}  // namespace

namespace ktanh_q8 {

// One launch's rows and channels, with a second launch for the sums of parts.
static ktanh_status_t launch_piece(const Operands &a, const Plan &plan, Way way, bool aligned, bool roomy, bool out_f32, void *workspace, ktanh_stream_t stream)
{
    if (way == TILES) {
        auto tiled = [&](const Operands &to, auto out) {
            constexpr Out O = decltype(out)::value;
            auto launch = [&](auto kernel) {
                const Tile t = kTiles[plan.kind];
                const unsigned over = (to.outer + t.over - 1) / t.over, across = (to.rows + t.across - 1) / t.across;
                return launch_checked(kernel, over * across * plan.parts, 256, stream, to, over, across, plan.parts);
            };
            if constexpr (O != SUMS) {
                if (plan.kind == T256) return launch(q8_tile_kernel<256, 256, 2, O>);
                if (plan.kind == T192) return launch(q8_tile_kernel<192, 256, 2, O>);
            }
            switch (plan.kind) {
            // a third place where a CU has no second block anyway: 1024 x 4096 x 4096 26.3 us, 34.8 with two
            case T128: return roomy ? launch(q8_tile_kernel<128, 128, 3, O>) : launch(q8_tile_kernel<128, 128, 2, O>);
            case T128_64: return launch(q8_tile_kernel<128, 64, 3, O>);
            case T128_32: return launch(q8_tile_kernel<128, 32, 3, O>);
            default: return launch(q8_tile_kernel<64, 64, 4, O>);
            }
        };
        if (plan.parts == 1) return out_f32 ? tiled(a, std::integral_constant<Out, F32>()) : tiled(a, std::integral_constant<Out, BF16>());
        Operands sums = a;
        sums.out = workspace;
        sums.out_row = a.outer;
        const ktanh_status_t st = tiled(sums, std::integral_constant<Out, SUMS>());
        if (st != KT_OK) return st;
        auto join = [&](auto kernel, unsigned each) {
            const unsigned long long chunks = (unsigned long long)((a.outer + each - 1) / each) * a.rows;
            return launch_checked(kernel, (unsigned)((chunks + 255) / 256), 256, stream, a, static_cast<const int *>(workspace), plan.parts);
        };
        return out_f32 ? join(q8_join_kernel<F32>, 4) : join(q8_join_kernel<BF16>, 8);
    }
    auto launch = [&](auto kernel, unsigned threads, unsigned each) {
        Operands to = a;
        void *args[] = {&to};
        return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((a.outer + each - 1) / each, (a.rows + each - 1) / each), dim3(threads), args, 0,
                               static_cast<hipStream_t>(stream)) == hipSuccess ? KT_OK : KT_ERR_HIP;
    };
    auto sized = [&](auto out_type, auto on_grid) {
        constexpr Out O = decltype(out_type)::value;
        constexpr bool A = decltype(on_grid)::value;
        return way == SHARED16 ? launch(q8_shared_inner_kernel<16, 16, 8, O, A>, 512, 16) : launch(q8_shared_inner_kernel<64, 64, 4, O, A>, 256, 64);
    };
    auto typed = [&](auto out_type) { return aligned ? sized(out_type, std::true_type()) : sized(out_type, std::false_type()); };
    return out_f32 ? typed(std::integral_constant<Out, F32>()) : typed(std::integral_constant<Out, BF16>());
}

// Arguments have been checked.
ktanh_status_t launch_product(const kq8_shape_t &s, const int8_t *x, size_t x_row, const float *x_scale, const int8_t *w, const float *w_scale,
                              const float *bias, void *out, void *workspace, ktanh_stream_t stream)
{
    Operands a;
    a.x_row = stride(s.rows, x_row);
    a.w_row = stride(s.outer, s.w_row);
    a.out_row = stride(s.rows, s.out_row);
    a.inner = (unsigned)s.inner;
    const bool aligned = !off(x, 16) && a.x_row % 16 == 0 && !off(w, 16) && a.w_row % 16 == 0;
    const Plan plan = plan_of(s.rows, s.inner, s.outer);
    const Way way = way_of(plan, s.rows, s.outer, aligned, a.x_row, a.w_row);
    const bool roomy = blocks_of(T128, s.rows, s.outer, plan.parts) <= 256;
    const Piece piece = piece_of(way, plan, s.rows, s.outer);
    for (size_t t = 0; t < s.rows; t += piece.rows)
        for (size_t o = 0; o < s.outer; o += piece.outer) {
            a.rows = (unsigned)(s.rows - t < piece.rows ? s.rows - t : piece.rows);
            a.outer = (unsigned)(s.outer - o < piece.outer ? s.outer - o : piece.outer);
            a.x = x + t * a.x_row;
            a.x_scale = x_scale + t;
            a.w = w + o * a.w_row;
            a.w_scale = w_scale + o;
            a.bias = bias != nullptr ? bias + o : nullptr;
            a.out = static_cast<char *>(out) + (t * a.out_row + o) * (s.out_f32 ? sizeof(float) : sizeof(uint16_t));
            const ktanh_status_t st = launch_piece(a, plan, way, aligned, roomy, s.out_f32 != 0, workspace, stream);
            if (st != KT_OK) return st;
        }
    return KT_OK;
}

}  // namespace ktanh_q8

namespace {

// What a product needs besides its rows.
ktanh_status_t check_weights(const kq8_shape_t *s, const int8_t *w, const float *w_scale, const float *bias, const void *out)
{
    if (w_scale == nullptr || out == nullptr || (s->inner != 0 && w == nullptr)) return KT_ERR_NULL;
    if (off(w_scale, 4) || off(bias, 4) || off(out, s->out_f32 ? 4 : 2)) return KT_ERR_ALIGN;
    return KT_OK;
}

// Whether a product's results share no memory with what it reads: x of x_size bytes an element, weights, scales, bias.
bool out_apart(const kq8_shape_t &s, const void *x, size_t x_size, const float *scales, const int8_t *w, const float *w_scale, const float *bias, const void *out)
{
    const Memory to = matrix(out, s.rows, s.outer, stride(s.rows, s.out_row), s.out_f32 ? 4 : 2);
    return apart(to, matrix(x, s.rows, s.inner, stride(s.rows, s.x_row), x_size)) && apart(to, matrix(w, s.outer, s.inner, stride(s.outer, s.w_row), 1)) &&
           apart(to, vector(scales, s.rows * sizeof(float))) && apart(to, vector(w_scale, s.outer * sizeof(float))) && apart(to, vector(bias, s.outer * sizeof(float)));
}

ktanh_status_t check_table(const ktanh_lut_t *lut) { return lut == nullptr ? KT_OK : ktanh_lut_validate(lut); }
ktanh_status_t check_table(const ktanh_lut64_t *lut) { return lut == nullptr ? KT_OK : ktanh_lut64_validate(lut); }

// Few short rows go to integers within the product's launch (ktanh_q8_few.hip).
ktanh_status_t launch_few(const kq8_shape_t &s, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out, const ktanh_lut_t *lut,
                          ktanh_stream_t stream, bool *done)
{
    return ktanh_q8::launch_few(s, x, w, w_scale, bias, out, lut, nullptr, false, stream, done);
}
ktanh_status_t launch_few(const kq8_shape_t &s, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out, const ktanh_lut64_t *lut,
                          ktanh_stream_t stream, bool *done)
{
    return ktanh_q8::launch_few(s, x, w, w_scale, bias, out, nullptr, lut, true, stream, done);
}

template <class Lut>
ktanh_status_t linear_entry(const kq8_shape_t *s, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out, void *workspace,
                            const Lut *lut, ktanh_stream_t stream)
{
    ktanh_status_t st = check_rows(s);
    if (st == KT_OK) st = check_product(s);
    if (st != KT_OK) return st;
    if (s->rows == 0 || s->outer == 0) return KT_OK;
    if (workspace == nullptr || (s->inner != 0 && x == nullptr)) return KT_ERR_NULL;
    st = check_weights(s, w, w_scale, bias, out);
    if (st != KT_OK) return st;
    if (off(x, s->x_f32 ? 4 : 2) || off(workspace, 16)) return KT_ERR_ALIGN;
    if (!out_apart(*s, x, s->x_f32 ? 4 : 2, nullptr, w, w_scale, bias, out)) {
        st = s->activation == KQ8_NONE ? KT_OK : check_table(lut);
        return st != KT_OK ? st : KT_ERR_SHAPE;
    }
    bool done = false;
    st = launch_few(*s, x, w, w_scale, bias, out, lut, stream, &done);
    if (done) return st;
    int8_t *codes = static_cast<int8_t *>(workspace);
    const size_t row = padded(s->inner);
    float *scales = reinterpret_cast<float *>(codes + s->rows * row);
    if constexpr (is_wide(static_cast<const Lut *>(nullptr))) st = kq8_rows64(s, x, codes, row, scales, lut, stream);
    else st = kq8_rows(s, x, codes, row, scales, lut, stream);
    if (st != KT_OK) return st;
    void *const sums = codes + rows_bytes(*s);
    return launch_product(*s, codes, row, scales, w, w_scale, bias, out, sums, stream);
}

}  // namespace

extern "C" ktanh_status_t kq8_product(const kq8_shape_t *shape, const int8_t *codes, const float *scales, const int8_t *w, const float *w_scale,
                                      const float *bias, void *out, void *workspace, ktanh_stream_t stream)
{
    ktanh_status_t st = check_product(shape);
    if (st != KT_OK) return st;
    if (shape->rows == 0 || shape->outer == 0) return KT_OK;
    if (scales == nullptr || (shape->inner != 0 && codes == nullptr)) return KT_ERR_NULL;
    st = check_weights(shape, w, w_scale, bias, out);
    if (st != KT_OK) return st;
    if (off(scales, 4) || off(workspace, 16)) return KT_ERR_ALIGN;
    if (workspace == nullptr && sums_bytes(*shape) != 0) return KT_ERR_NULL;
    if (!out_apart(*shape, codes, 1, scales, w, w_scale, bias, out)) return KT_ERR_SHAPE;
    return launch_product(*shape, codes, shape->x_row, scales, w, w_scale, bias, out, workspace, stream);
}

extern "C" size_t kq8_product_workspace(const kq8_shape_t *shape) { return check_product(shape) != KT_OK ? 0 : sums_bytes(*shape); }

extern "C" size_t kq8_linear_workspace(const kq8_shape_t *shape)
{
    if (check_rows(shape) != KT_OK || check_product(shape) != KT_OK) return 0;
    return rows_bytes(*shape) + sums_bytes(*shape);
}

extern "C" ktanh_status_t kq8_linear(const kq8_shape_t *shape, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out,
                                     void *workspace, const ktanh_lut_t *lut, ktanh_stream_t stream)
{
    return linear_entry(shape, x, w, w_scale, bias, out, workspace, lut, stream);
}
extern "C" ktanh_status_t kq8_linear64(const kq8_shape_t *shape, const void *x, const int8_t *w, const float *w_scale, const float *bias, void *out,
                                       void *workspace, const ktanh_lut64_t *lut, ktanh_stream_t stream)
{
    return linear_entry(shape, x, w, w_scale, bias, out, workspace, lut, stream);
}
