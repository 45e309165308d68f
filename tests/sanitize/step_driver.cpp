// Host code of the verification step's C ABI (csrc/ciar_step.cpp) on a machine without a GPU, under the sanitizers: every "device"
// pointer is host memory of exactly the documented size, and the stand-in launchers write the full extent that the kernels may write
// (and read the ends of what they may read): a size or a stride that the checks let through wrongly is a heap overflow that the
// sanitizer reports.  Random calls, most of them valid; an invalid one must come back without a launch.
#include "../../include/ciar.h"
#include "../../paper_2603_25463_amd/csrc/ciar_step.h"

#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <thread>
#include <vector>

static std::atomic<int> launches{0}, failed{0};
#define EXPECT(x) do { if (!(x)) { ++failed; std::printf("line %d: %s (%s)\n", __LINE__, #x, ciar_last_error()); } } while (0)

namespace {
thread_local volatile char sink;
void touch(void* p, size_t n) { if (p && n) std::memset(p, 0x5a, n); }
void look(const void* p, size_t n) { if (p && n) { sink = static_cast<const char*>(p)[0]; sink = static_cast<const char*>(p)[n - 1]; } }
void touch_heads(const ciar::Heads& h, int64_t T, int heads, int D, int elt)
{
    for (int64_t t = 0; t < T; ++t)
        for (int i = 0; i < heads; ++i) touch((char*)h.p + (t * h.token + i * h.head) * elt, (size_t)D * elt);
}
void look_heads(const ciar::Heads& h, int64_t T, int heads, int D, int elt)
{
    if (T > 0) { look(h.p, 1); look((const char*)h.p + ((T - 1) * h.token + (heads - 1) * h.head + D - 1) * elt, (size_t)elt); }
}
}  // namespace

namespace ciar {
hipError_t launch_plan(const PlanArgs& a, hipStream_t)
{
    ++launches;
    look(a.lengths, 4u * a.R); look(a.kept, 4u * a.R); look(a.fresh, 4u * a.R); look(a.held, 4u * a.R); look(a.ring_state, 16);
    touch(a.ring, 4u * a.P);
    for (int r = 0; r < a.R; ++r) touch(a.table + r * a.table_stride, 4u * a.width);
    touch(a.out_lengths, 4u * a.R); touch(a.kv_len, 4u * a.R); touch(a.cu_new, 4u * (a.R + 1)); touch(a.out_held, 4u * a.R);
    touch(a.granted, (size_t)a.R); touch(a.out_ring_state, 16);
    touch(a.slots, 4u * a.T); touch(a.positions, 4u * a.T); touch(a.requests, 4u * a.T);
    return hipSuccess;
}
hipError_t launch_rotary(int dtype, bool, const RotaryArgs& a, hipStream_t)
{
    ++launches;
    const int elt = dtype == 0 ? 4 : 2;
    look_heads(a.q, a.T, a.q_heads, a.D, elt);
    look_heads(a.k, a.T, a.kv_heads, a.D, elt);
    look(a.positions, 4u * a.T); look(a.inv_freq, 4u * a.n);
    touch_heads(a.q_out, a.T, a.q_heads, a.D, elt);
    if (a.k_cache) {
        look_heads(a.v, a.T, a.kv_heads, a.D, elt);
        look(a.slots, 4u * a.T);
        touch(a.k_cache, (size_t)a.slot_count * a.kv_heads * a.D * 2);
        touch(a.v_cache, (size_t)a.slot_count * a.kv_heads * a.D * 2);
    } else touch_heads(a.k_out, a.T, a.kv_heads, a.D, elt);
    return hipSuccess;
}
size_t attention_workspace(const AttentionArgs& a) { return a.max_len > 64 ? 3 * (size_t)a.T * a.q_heads * (a.D * 4 + 8) : 0; }
hipError_t launch_attention(const AttentionArgs& a, void* ws, hipStream_t)
{
    ++launches;
    look_heads(a.q, a.T, a.q_heads, a.D, 2);
    look(a.cu_new, 4u * (a.R + 1)); look(a.kv_len, 4u * a.R);
    if (a.R > 0) look(a.table, 4u * ((a.R - 1) * a.table_stride + a.width));
    look(a.k_cache, (size_t)a.pages * a.page * a.kv_heads * a.D * 2); look(a.v_cache, (size_t)a.pages * a.page * a.kv_heads * a.D * 2);
    touch_heads(a.out, a.T, a.q_heads, a.D, 2);
    touch(a.lse, 4u * (size_t)a.T * a.q_heads);
    touch(ws, attention_workspace(a));
    EXPECT(a.max_len <= (int64_t)a.width * a.page && a.max_new <= a.T);
    return hipSuccess;
}
hipError_t launch_adjust(int dtype, LogitArgs a, hipStream_t)
{
    ++launches;
    const size_t elt = dtype == 0 ? 4 : 2, per = 16 / elt;
    const int64_t W = (a.N + a.window - 1) / a.window;
    look(a.logits, ((a.N - 1) * a.stride + (a.V + per - 1) / per * per) * elt);
    for (int64_t n = 0; n < a.N; ++n) touch((char*)a.out + n * a.out_stride * elt, a.V * elt);
    touch(a.left, 4u * a.N); touch(a.left_words, 8u * a.N);
    look(a.history_start, a.history_start ? 8u * (W + 1) : 0); look(a.history, 4u * a.history_len); look(a.prompt_len, a.prompt_len ? 4u * W : 0);
    look(a.drafted, a.drafted ? 4u * a.N : 0); look(a.repetition, a.repetition ? 4u * W : 0); look(a.bias_ids, 4u * a.bias_len);
    look(a.allowed, a.allowed ? 4u * ((a.mask_rows - 1) * a.allowed_stride + (a.V + 31) / 32) : 0);
    look(a.allowed_row, a.allowed ? 4u * a.N : 0);
    EXPECT(a.tag != 0 && (a.left != nullptr) == (a.left_words != nullptr));
    return hipSuccess;
}
}  // namespace ciar

namespace {
struct Buf {
    void* p;
    explicit Buf(size_t n) : p(std::aligned_alloc(16, n ? (n + 15) / 16 * 16 : 16)) { std::memset(p, 0, n ? n : 1); }
    ~Buf() { std::free(p); }
    Buf(const Buf&) = delete;
    template <class T> T* as() const { return static_cast<T*>(p); }
};

void plans(unsigned seed)
{
    std::mt19937 g(seed);
    for (int i = 0; i < 200; ++i) {
        const int64_t R = g() % 9, T = g() % 40, P = 1 + g() % 30, width = 1 + g() % 6, stride = width + g() % 3;
        Buf l(4 * R), k(4 * R), n(4 * R), h(4 * R), ring(4 * P), st(16), tab(R ? 4 * ((R - 1) * stride + width) : 0), ol(4 * R), kv(4 * R),
            cu(4 * (R + 1)), oh(4 * R), gr(R), os(16), sl(4 * T), po(4 * T), rq(4 * T);
        const int page = i % 10 == 9 ? 20 : 16 * (1 + g() % 3), before = launches;
        const int rc = ciar_cache_plan(l.as<int32_t>(), g() % 2 ? k.as<int32_t>() : nullptr, n.as<int32_t>(), h.as<int32_t>(), R, ring.as<int32_t>(), P,
                                       st.as<int64_t>(), tab.as<int32_t>(), (int32_t)width, stride, page, T, ol.as<int32_t>(), kv.as<int32_t>(),
                                       cu.as<int32_t>(), oh.as<int32_t>(), gr.as<uint8_t>(), os.as<int64_t>(), sl.as<int32_t>(), po.as<int32_t>(),
                                       rq.as<int32_t>(), nullptr);
        EXPECT(rc == (page % 16 ? CIAR_EUNSUPPORTED : CIAR_OK));
        if (rc && seed == 1) EXPECT(launches == before);
    }
}

void rotaries(unsigned seed)
{
    std::mt19937 g(seed);
    for (int i = 0; i < 200; ++i) {
        const bool cached = g() % 2;
        ciar_rotary_params p = {};
        p.struct_size = sizeof p;
        p.dtype = cached ? CIAR_BF16 : (int)(g() % 2);
        const int elt = p.dtype == CIAR_F32 ? 4 : 2;
        p.q_heads = 1 + g() % 5; p.kv_heads = 1 + g() % 3;
        p.head_dim = cached ? 8 * (1 + g() % 4) : 2 + g() % 30;
        p.rotary_dim = 2 * (1 + g() % (p.head_dim / 2));
        p.interleaved = g() % 2; p.inverse = g() % 2; p.magnitude = 1.5;
        p.page_size = 16 * (1 + g() % 2); p.cache_pages = 1 + g() % 4;
        const int64_t T = g() % 12, D = p.head_dim, inner = D + g() % 3;
        // heads of a token side by side, or tokens of a head
        const bool outer = g() % 2;
        auto lay = [&](int64_t heads, int64_t& token, int64_t& head) {
            token = outer ? inner : heads * inner + 1;
            head = outer ? (T > 0 ? T : 1) * inner + 2 : inner;
        };
        lay(p.q_heads, p.q_stride, p.q_head_stride);
        lay(p.kv_heads, p.k_stride, p.k_head_stride);
        lay(p.kv_heads, p.v_stride, p.v_head_stride);
        lay(p.q_heads, p.q_out_stride, p.q_out_head_stride);
        lay(p.kv_heads, p.k_out_stride, p.k_out_head_stride);
        auto bytes = [&](int64_t token, int64_t head, int64_t heads) { return (size_t)(T ? ((T - 1) * token + (heads - 1) * head + D) * elt : 0); };
        const size_t cb = (size_t)p.cache_pages * p.page_size * p.kv_heads * D * 2;
        Buf q(bytes(p.q_stride, p.q_head_stride, p.q_heads)), k(bytes(p.k_stride, p.k_head_stride, p.kv_heads)), v(bytes(p.v_stride, p.v_head_stride, p.kv_heads)),
            qo(bytes(p.q_out_stride, p.q_out_head_stride, p.q_heads)), ko(bytes(p.k_out_stride, p.k_out_head_stride, p.kv_heads)), pos(4 * T),
            fr(4 * p.rotary_dim), kc(cb), vc(cb), sl(4 * T);
        const int rc = ciar_rotary(q.p, k.p, cached ? v.p : nullptr, pos.as<int32_t>(), fr.as<double>(), T, &p, qo.p, cached ? nullptr : ko.p,
                                   cached ? kc.p : nullptr, cached ? vc.p : nullptr, cached ? sl.as<int32_t>() : nullptr, nullptr);
        EXPECT(rc == CIAR_OK);
        p.q_out_head_stride = D - 1;
        if (T > 0 && p.q_heads > 1)
            EXPECT(ciar_rotary(q.p, k.p, cached ? v.p : nullptr, pos.as<int32_t>(), fr.as<double>(), T, &p, qo.p, cached ? nullptr : ko.p,
                               cached ? kc.p : nullptr, cached ? vc.p : nullptr, cached ? sl.as<int32_t>() : nullptr, nullptr) == CIAR_EINVAL);
    }
}

void attentions(unsigned seed)
{
    std::mt19937 g(seed);
    for (int i = 0; i < 200; ++i) {
        ciar_attention_params p = {};
        p.struct_size = sizeof p;
        p.kv_heads = 1 + g() % 3; p.q_heads = p.kv_heads * (1 + g() % 3);
        p.head_dim = 32 * (1 + g() % 8); p.page_size = 16 * (1 + g() % 2); p.table_width = 1 + g() % 8;
        p.max_new = g() % 20; p.max_len = g() % 300; p.scale = 0.1f;
        p.table_stride = p.table_width + g() % 2; p.cache_pages = 1 + g() % 5;
        const int64_t T = g() % 20, R = g() % 4, D = p.head_dim;
        p.q_stride = p.out_stride = p.q_heads * D + 3; p.q_head_stride = p.out_head_stride = D;
        const size_t rows = T ? ((T - 1) * p.q_stride + p.q_heads * D) * 2 : 0, cb = (size_t)p.cache_pages * p.page_size * p.kv_heads * D * 2;
        const size_t need = ciar_attention_workspace_bytes(R, T, &p);
        Buf q(rows), o(rows), lse(4 * T * p.q_heads), kc(cb), vc(cb), tab(R ? 4 * ((R - 1) * p.table_stride + p.table_width) : 0), cu(4 * (R + 1)), kl(4 * R),
            ws(need);
        // (without requests nothing is split: the stand-in asks for a workspace all the same, by the call's sizes)
        const size_t given = R > 0 ? need : (size_t)1 << 20;
        Buf more(R > 0 ? 0 : given);
        const int rc = ciar_paged_attention(q.p, kc.p, vc.p, tab.as<int32_t>(), cu.as<int32_t>(), kl.as<int32_t>(), R, T, &p, o.p,
                                            g() % 2 ? lse.as<float>() : nullptr, R > 0 ? ws.p : more.p, given, nullptr);
        EXPECT(rc == CIAR_OK);
        if (need && T > 0)
            EXPECT(ciar_paged_attention(q.p, kc.p, vc.p, tab.as<int32_t>(), cu.as<int32_t>(), kl.as<int32_t>(), R, T, &p, o.p, nullptr, ws.p, need - 256,
                                        nullptr) == CIAR_EWORKSPACE);
    }
}

void adjustments(unsigned seed)
{
    std::mt19937 g(seed);
    for (int i = 0; i < 200; ++i) {
        ciar_params p;
        ciar_params_default(&p);
        p.dtype = (int)(g() % 2);
        const int elt = p.dtype == CIAR_F32 ? 4 : 2, per = 16 / elt;
        p.vocab = 1 + g() % 200; p.window = 1 + g() % 9;
        p.row_stride = (p.vocab + per - 1) / per * per + per * (int)(g() % 2);
        const int64_t N = g() % 20, W = (N + p.window - 1) / p.window, os = (p.vocab + per - 1) / per * per, words = (p.vocab + 31) / 32;
        const size_t whole = N ? ((N - 1) * p.row_stride + (p.vocab + per - 1) / per * per) * elt : 0, need = ciar_adjust_workspace_bytes(N, &p);
        Buf x(whole), y(N ? ((N - 1) * os + p.vocab) * elt : 0), left(4 * N), ws(need), hs(8 * (W + 1)), hist(4 * 50), pl(4 * W), dr(4 * N), a(4 * W), b(4 * W),
            c(4 * W), bs(8 * (W + 1)), bi(4 * 7), bv(4 * 7), al(4 * 3 * words), ar(4 * N);
        ciar_adjustments j = {};
        j.struct_size = sizeof j;
        if (g() % 2) { j.history_start = hs.as<int64_t>(); j.history = hist.as<int32_t>(); j.history_len = 50; if (g() % 2) j.prompt_len = pl.as<int32_t>(); }
        if (g() % 2) j.drafted = dr.as<int32_t>();
        if (g() % 2) { j.repetition = a.as<float>(); j.presence = b.as<float>(); j.frequency = c.as<float>(); }
        if (g() % 2) { j.bias_start = bs.as<int64_t>(); j.bias_ids = bi.as<int32_t>(); j.bias_values = bv.as<float>(); j.bias_len = 7; }
        if (g() % 2) { j.allowed = al.as<int32_t>(); j.mask_rows = 3; j.allowed_stride = words; j.allowed_row = ar.as<int32_t>(); }
        const bool count = g() % 2, same = g() % 2;
        const int rc = ciar_adjust_logits(x.p, N, &p, &j, same ? x.p : y.p, same ? p.row_stride : os, count ? left.as<int32_t>() : nullptr,
                                          count ? ws.p : nullptr, count ? need : 0, nullptr);
        EXPECT(rc == CIAR_OK);
        if (count && N > 0)
            EXPECT(ciar_adjust_logits(x.p, N, &p, &j, y.p, os, left.as<int32_t>(), ws.p, need - 8, nullptr) == CIAR_EWORKSPACE);
    }
}
}  // namespace

int main()
{
    plans(1); rotaries(2); attentions(3); adjustments(4);
    std::vector<std::thread> t;
    for (unsigned s = 10; s < 14; ++s) t.emplace_back([s] { plans(s); rotaries(s); attentions(s); adjustments(s); });
    for (auto& x : t) x.join();
    std::printf("%d launches, %d failed expectations\n", launches.load(), failed.load());
    return failed ? 1 : 0;
}
