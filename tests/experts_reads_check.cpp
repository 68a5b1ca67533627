// Where the experts' kernels read by buffer, on the host: every load that may reach memory lies inside its tensor.
//   experts_reads_check dw TYPE TILE J K lddy before rows behind      two experts with rows, and rows that nobody has behind them
//   experts_reads_check dx TYPE TILE rows N K lddy                     one expert
//   experts_reads_check few N K M blocks                               a layer of few rows, from codes and, of up to 4096 values, quantised on the way
//   experts_reads_check gemm TILE N K rows rows                        two experts, and the last of the weights' rows; plain, and with a bias, a residual and a kept form
// Prints "ok <loads>" or what lies outside.  A load's offset has two parts.  Which of them meets the buffer's size is told in two ways: the vector part alone; or the
// vector part against the size less the scalar part, in 32 bits without a sign.  A load that either of them lets through may reach memory.
#define __shared__
#include <sys/mman.h>
#include <stdio.h>
#include <stdlib.h>

#include "../paper_2105_11010_amd/csrc/sparq_mx_experts_grad.h"
#include "../paper_2105_11010_amd/csrc/sparq_mx_experts_gemm.h"

using namespace sparq::mx;

namespace sparq {
namespace mx {
alignas(16) uint8_t lds8[160 * 1024], lds[160 * 1024];
}  // namespace mx
}  // namespace sparq

// A tensor that ends where its pages do: an ordinary load behind it ends the check.
struct Tensor {
    uint8_t *begin, *end;
    explicit Tensor(size_t bytes) {
        const size_t pages = (bytes + 4095) / 4096 * 4096;
        uint8_t* const p = static_cast<uint8_t*>(mmap(nullptr, pages + 4096, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
        if (p == MAP_FAILED || mprotect(p + pages, 4096, PROT_NONE)) exit(3);
        end = p + pages;
        begin = end - bytes;
    }
};
static std::vector<Tensor> tensors;
static long loads, outside;

void gpu::load(const Buffer& b, uint32_t vector, uint32_t scalar, int bytes) {
    ++loads;
    for (int at = 0; at < bytes; at += bytes < 4 ? bytes : 4) {          // (a load is checked word by word)
        const uint32_t v = vector + at;
        if (v >= b.bytes && v >= b.bytes - scalar) continue;
        const uint8_t *from = b.base + v + (uint64_t)scalar, *to = from + (bytes < 4 ? bytes : 4);
        bool inside = false;
        for (const Tensor& t : tensors) inside |= b.base >= t.begin && b.base <= t.end && from >= t.begin && to <= t.end;
        if (!inside && ++outside <= 5) printf("outside: vector offset %u, scalar offset %u, size %u\n", v, scalar, b.bytes);
    }
}

template <class T, int TILE>
static void dw(int64_t J, int K, int64_t lddy, int rows_before, int rows, int behind) {
    constexpr int kAll = 20;                     // experts
    const int64_t M = (int64_t)rows_before + rows + behind;
    Tensor dy(((M - 1) * lddy + J) * sizeof(T)), codes(M * code_pitch(K, 8)), scales(M * scale_pitch(K)), out(kAll * J * K * 4);
    tensors = {dy, codes, scales};
    std::vector<int32_t> offsets(kAll + 1, rows_before);
    offsets[0] = 0;
    offsets[kAll] = rows_before + rows;
    ExpertGradParams p = {};
    p.dy = dy.begin;
    p.codes = codes.begin;
    p.scales = scales.begin;
    p.lddy = lddy;
    p.code_pitch = code_pitch(K, 8);
    p.scale_pitch = scale_pitch(K);
    p.ldo = K;
    p.J = J;
    p.K = K;
    p.K128 = (int)sparq::round_up(K, kCodeUnit);
    p.offsets = offsets.data();
    p.rows = M;
    p.experts = kAll;
    p.tiles_j = (int)((J + TILE - 1) / TILE);
    p.tiles_k = (K + TILE - 1) / TILE;
    p.margin = (int)((sparq::round_up(J, 8) - J + lddy - 1) / lddy);
    for (int expert : {0, kAll - 1})
        for (int block = 0; block < p.tiles_j * p.tiles_k; ++block)
            gpu::run_threads(kGradThreads, dim3(block, expert), [&] { grad_wide_kernel<T, float, true, TILE, ExpertGradParams>(reinterpret_cast<float*>(out.begin), p); });
}

template <class T, int TILE>
static void dx(int rows, int N, int K, int64_t lddy) {
    Tensor dy(((rows - 1) * lddy + N) * sizeof(T)), codes(N * code_pitch(K, 4)), scales(N * scale_pitch(K)), out((int64_t)rows * K * 4), table(sizeof(ExpertTile) * (rows / 64 + 2));
    tensors = {dy, codes, scales};
    ExpertTile* const t = reinterpret_cast<ExpertTile*>(table.begin);
    t[0].row = (rows + TILE - 1) / TILE;
    for (int i = 0; i < t[0].row; ++i) t[1 + i] = {i * TILE, rows - i * TILE < TILE ? rows - i * TILE : TILE, 0, 0};
    ExpertGradParams p = {};
    p.dy = dy.begin;
    p.codes = codes.begin;
    p.scales = scales.begin;
    p.lddy = lddy;
    p.code_pitch = code_pitch(K, 4);
    p.scale_pitch = scale_pitch(K);
    p.ldo = K;
    p.R = N;
    p.K = K;
    p.K128 = (int)sparq::round_up(K, kCodeUnit);
    p.table = t;
    p.rows = rows;
    p.experts = 1;
    p.tiles_k = (K + TILE - 1) / TILE;
    p.s_whole = N / kGradStep;
    p.steps_per_part = (N + kGradStep - 1) / kGradStep;
    for (int block = 0; block < t[0].row * p.tiles_k; ++block)
        gpu::run_threads(kGradThreads, dim3(block), [&] { grad_wide_kernel<T, float, false, TILE, ExpertGradParams>(reinterpret_cast<float*>(out.begin), p); });
}
// The kernels that there are: tiles of 256 for bf16 alone
template <class F>
static void with_kernel(const char* type, int tile, F&& f) {
    typedef std::integral_constant<int, 64> Small;
    typedef std::integral_constant<int, 128> Middle;
    if (!strcmp(type, "f32")) tile == 128 ? f(float{}, Middle{}) : f(float{}, Small{});
    else if (!strcmp(type, "f16")) tile == 128 ? f(_Float16{}, Middle{}) : f(_Float16{}, Small{});
    else if (tile == 256) f(__bf16{}, std::integral_constant<int, 256>{});
    else tile == 128 ? f(__bf16{}, Middle{}) : f(__bf16{}, Small{});
}

template <class X, int WAVES, bool SINGLE>
static void few(int N, int K, int M, int blocks) {
    typedef std::conditional_t<std::is_void_v<X>, float, X> Value;
    const int64_t ldx = K + 3;
    Tensor x(((M - 1) * ldx + K) * sizeof(Value)), a(M * code_pitch(K, 4)), as(M * scale_pitch(K)), w(N * code_pitch(K, 4)), ws(N * scale_pitch(K)), y((int64_t)M * N * 4);
    tensors = {w, ws};
    ExpertFewParams p = {};
    p.x = x.begin;
    p.ldx = ldx;
    p.a = a.begin;
    p.as = as.begin;
    p.w = w.begin;
    p.ws = ws.begin;
    p.ldy = N;
    p.code_pitch = code_pitch(K, 4);
    p.scale_pitch = scale_pitch(K);
    p.M = M;
    p.N = N;
    p.K = K;
    p.groups = (K + kScaleUnit - 1) / kScaleUnit;
    p.last_step = (K + kCodeUnit - 1) / kCodeUnit - 1;
    p.experts = 1;
    p.blocks = blocks;
    p.epilogue.function = SPARQ_MX_NONE;
    const int all = (N + kFewColumns - 1) / kFewColumns;
    for (int block = 0; block < (all + blocks - 1) / blocks; ++block)
        gpu::run_threads(WAVES * 64, dim3(block), [&] { experts_few_kernel<float, X, 1, WAVES, SINGLE>(reinterpret_cast<float*>(y.begin), p); });
}

template <class O, int TILE>
static void gemm(int N, int K, int first, int second, bool epilogue) {
    const int64_t M = first + second;
    Tensor a(M * code_pitch(K, 4)), as(M * scale_pitch(K)), w(2 * N * code_pitch(K, 4)), ws(2 * N * scale_pitch(K)), y(M * N * sizeof(O));
    Tensor bias(2 * N * 4), residual(M * N * sizeof(O)), kept(M * code_pitch(N, 8)), kept_scales(M * scale_pitch(N));
    tensors = {a, as, w, ws};
    std::vector<ExpertTile> table(1);
    const int32_t offsets[] = {0, first, first + second};
    for (int e = 0; e < 2; ++e)
        for (int row = offsets[e]; row < offsets[e + 1]; row += TILE) table.push_back({row, offsets[e + 1] - row < TILE ? offsets[e + 1] - row : TILE, e, 0});
    table[0].row = (int)table.size() - 1;
    ExpertGemmParamsOf<SPARQ_MX_NONE> p = {};
    p.a = a.begin;
    p.as = as.begin;
    p.w = w.begin;
    p.ws = ws.begin;
    p.M = M;
    p.N = N;
    p.ldy = N;
    p.code_pitch = (uint32_t)code_pitch(K, 4);
    p.scale_pitch = (uint32_t)scale_pitch(K);
    p.tiles_m = (uint32_t)most_tiles(M, 2, TILE);
    p.tiles_n = (uint32_t)((N + TILE - 1) / TILE);
    p.steps = p.steps_per_part = (int)sparq::round_up((K + kCodeUnit - 1) / kCodeUnit, 4);
    p.items = p.tiles_m * p.tiles_n;
    p.table = table.data();
    p.offsets = offsets;
    p.experts = 2;
    p.epilogue = {nullptr, nullptr, nullptr, N, code_pitch(N, 8), scale_pitch(N), SPARQ_MX_NONE, (int)sparq::round_up(N, kCodeUnit)};
    if (epilogue) {
        p.bias = reinterpret_cast<const float*>(bias.begin);
        p.epilogue.residual = residual.begin;
        p.epilogue.kept_codes = kept.begin;
        p.epilogue.kept_scales = kept_scales.begin;
    }
    gridDim = dim3(2);                           // (workgroups that take one tile after the other)
    for (int block = 0; block < 2; ++block)
        gpu::run_threads(kGemmThreads, dim3(block), [&] { gemm_kernel<O, TILE, TILE, ExpertGemmParamsOf<SPARQ_MX_NONE>>(reinterpret_cast<O*>(y.begin), p); });
}

int main(int argc, char** argv) {
    std::vector<int> n;
    for (int i = 0; i < argc; ++i) n.push_back(atoi(argv[i]));
    if (argc == 10 && !strcmp(argv[1], "dw")) {
        with_kernel(argv[2], n[3], [&](auto t, auto tile) { dw<decltype(t), decltype(tile)::value>(n[4], n[5], n[6], n[7], n[8], n[9]); });
    } else if (argc == 8 && !strcmp(argv[1], "dx")) {
        with_kernel(argv[2], n[3], [&](auto t, auto tile) { dx<decltype(t), decltype(tile)::value>(n[4], n[5], n[6], n[7]); });
    } else if (argc == 6 && !strcmp(argv[1], "few")) {
        const int groups = (n[3] + kScaleUnit - 1) / kScaleUnit;
        (groups <= 4 ? few<void, 4, true> : groups <= 8 ? few<void, 8, true> : few<void, 8, false>)(n[2], n[3], n[4], n[5]);
        if (groups <= 8) {
            (groups <= 4 ? few<float, 4, true> : few<float, 8, true>)(n[2], n[3], n[4], n[5]);
            (groups <= 4 ? few<__bf16, 4, true> : few<__bf16, 8, true>)(n[2], n[3], n[4], n[5]);
        }
    } else if (argc == 7 && !strcmp(argv[1], "gemm")) {
        for (const bool epilogue : {false, true}) {
            (n[2] == 256 ? gemm<float, 256> : n[2] == 128 ? gemm<float, 128> : gemm<float, 64>)(n[3], n[4], n[5], n[6], epilogue);
            (n[2] == 256 ? gemm<__bf16, 256> : n[2] == 128 ? gemm<__bf16, 128> : gemm<__bf16, 64>)(n[3], n[4], n[5], n[6], epilogue);
        }
    } else {
        return 2;
    }
    if (outside) return printf("%ld of %ld loads' words outside\n", outside, loads), 1;
    printf("ok %ld\n", loads);
    return 0;
}
