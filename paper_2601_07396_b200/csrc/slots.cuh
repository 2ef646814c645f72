// Which rows of a tile belong to which request of a product with adapters.  A slot is a pair of a tile and a request that have rows in
// common, tile + request its number: along the rows one of both grows from each pair to the next, so no two pairs share one.
//
// A warp walks over the requests, 32 at a time.  The walks are written on what a warp can do (Warp), so that the same code runs on
// the host (OneThread, which stands for all lanes) in tests.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace svdc {

// the requests of a call as the kernels see them, in tiles of 1 << tile_shift rows
struct Requests {
    const int32_t *row_start, *adapter;
    int64_t first, M;                                // the rows that a launch computes: [first, first + M) of the caller's
    int requests, count, tile_shift;
    // first row of request i (the end for i = requests), counted from the launch's first
    __host__ __device__ __forceinline__ int row(int i) const {
        const int64_t r = row_start[i] - first;
        return r < 0 ? 0 : r > M ? (int)M : (int)r;
    }
};
struct Run { int lo, hi, adapter; };                 // a request's rows; the adapter -1 beyond the last request

__host__ __device__ __forceinline__ int how_many(uint32_t lanes) {
#ifdef __CUDA_ARCH__
    return __popc(lanes);
#else
    return __builtin_popcount(lanes);
#endif
}
struct Warp {
    int lane;
    template <typename T> struct Of { T v; };
    template <typename T, typename F> __device__ __forceinline__ Of<T> each(F f) const { return {f(lane)}; }
    template <typename T, typename F> __device__ __forceinline__ uint32_t ballot(const Of<T> &o, F f) const { return __ballot_sync(0xFFFFFFFFu, f(lane, o.v)); }
    template <typename T> __device__ __forceinline__ int from(const Of<T> &o, int T::*member, int source) const { return __shfl_sync(0xFFFFFFFFu, o.v.*member, source); }
    template <typename T, typename F> __device__ __forceinline__ void where(uint32_t lanes, const Of<T> &o, F f) const {
        if (lanes >> lane & 1u) f(lane, o.v);
    }
    __device__ __forceinline__ bool leader() const { return lane == 0; }
    __device__ __forceinline__ int lowest(uint32_t lanes) const { return __ffs((int)lanes) - 1; }
    __device__ __forceinline__ int highest(uint32_t lanes) const { return 31 - __clz((int)lanes); }
};
struct OneThread {
    template <typename T> struct Of { T v[32]; };
    template <typename T, typename F> Of<T> each(F f) const {
        Of<T> o;
        for (int i = 0; i < 32; ++i) o.v[i] = f(i);
        return o;
    }
    template <typename T, typename F> uint32_t ballot(const Of<T> &o, F f) const {
        uint32_t lanes = 0;
        for (int i = 0; i < 32; ++i) lanes |= (uint32_t)(f(i, o.v[i]) ? 1u : 0u) << i;
        return lanes;
    }
    template <typename T> int from(const Of<T> &o, int T::*member, int source) const { return o.v[source].*member; }
    template <typename T, typename F> void where(uint32_t lanes, const Of<T> &o, F f) const {
        for (int i = 0; i < 32; ++i)
            if (lanes >> i & 1u) f(i, o.v[i]);
    }
    bool leader() const { return true; }
    int lowest(uint32_t lanes) const { return __builtin_ctz(lanes); }
    int highest(uint32_t lanes) const { return 31 - __builtin_clz(lanes); }
};

#pragma nv_exec_check_disable
template <typename W> __host__ __device__ __forceinline__ typename W::template Of<Run> runs_from(const W &w, const Requests &q, int i0) {
    return w.template each<Run>([&](int lane) {
        const int i = i0 + lane;
        const bool is = i < q.requests;
        return Run{is ? q.row(i) : 0, is ? q.row(i + 1) : 0, is ? q.adapter[i] : -1};
    });
}

// Calls sink(place, first slot, {slot, adapter}), a lane for each, for the slots of a tile that have an adapter, places counted from
// 0 and below `most`; returns how many there are, and in `first` the first one's slot and adapter.
#pragma nv_exec_check_disable
template <typename W, typename F> __host__ __device__ __forceinline__ int tile_slots_of(const W &w, const Requests &q, int tile, int most, int2 &first, F sink) {
    const int64_t row0 = (int64_t)tile << q.tile_shift, end = row0 + (1 << q.tile_shift);
    int slots = 0;
    first = make_int2(tile, 0);
    for (int i0 = 0; i0 < q.requests; i0 += 32) {
        const auto runs = runs_from(w, q, i0);
        const uint32_t with = w.ballot(runs, [&](int, const Run &r) { return r.lo < r.hi && r.lo < end && r.hi > row0 && r.adapter >= 0 && r.adapter < q.count; });
        if (!with) continue;
        const int source = w.lowest(with), a0 = w.from(runs, &Run::adapter, source);
        if (slots == 0) first = make_int2(tile + i0 + source, a0);
        w.where(with, runs, [&](int lane, const Run &r) {
            const int place = slots + how_many(with & ((1u << lane) - 1u));
            if (place < most) sink(place, first.x, make_int2(tile + i0 + lane, r.adapter));
        });
        slots += how_many(with);
    }
    return slots < most ? slots : most;
}

// A tile's slots into the lists of a call: where they are listed, how many they are, the first one's number and adapter; they are listed from the
// first one's number on, so no two tiles' lists meet.
#pragma nv_exec_check_disable
template <typename W> __host__ __device__ __forceinline__ void write_tile_slots(const W &w, const Requests &q, int tile, int4 *tile_slots, int2 *slot_list) {
    int2 first;
    const int slots = tile_slots_of(w, q, tile, 0x7FFFFFFF, first, [&](int place, int from, int2 slot) { slot_list[from + place] = slot; });
    if (w.leader()) tile_slots[tile] = make_int4(first.x, slots, first.x, first.y);
}

struct Task { int tile, lo, hi, adapter; };           // rows [lo, hi) of M; adapter < 0: none
// The pair that a slot belongs to: the last request whose own first slot is not behind it.  A lane reads all there is to a request at
// once: this stands before the first load of A.
#pragma nv_exec_check_disable
template <typename W> __host__ __device__ __forceinline__ Task find_task(const W &w, const Requests &q, int tiles, int slot) {
    Task t{0, 0, 0, -1};
    int s = -1, lo = 0, hi = 0, a = -1;
    for (int i0 = 0; i0 < q.requests; i0 += 32) {
        const auto runs = runs_from(w, q, i0);
        const uint32_t begun = w.ballot(runs, [&](int lane, const Run &r) { return i0 + lane < q.requests && (r.lo >> q.tile_shift) + i0 + lane <= slot; });
        if (!begun) break;
        const int source = w.highest(begun);
        s = i0 + source;
        lo = w.from(runs, &Run::lo, source);
        hi = w.from(runs, &Run::hi, source);
        a = w.from(runs, &Run::adapter, source);
        if (source != 31) break;
    }
    t.tile = slot - s;
    if (s < 0 || t.tile < 0 || t.tile >= tiles) return t;
    const int64_t row0 = (int64_t)t.tile << q.tile_shift, end = row0 + (1 << q.tile_shift);
    t.lo = (int)(lo > row0 ? lo : row0);
    t.hi = (int)(hi < end ? hi : end);
    if (t.lo < t.hi && a >= 0 && a < q.count) t.adapter = a;
    return t;
}

}  // namespace svdc
