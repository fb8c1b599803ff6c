// Whether outputs of a call overlap each other or its inputs, told exactly from addresses, sizes and strides (host only).
#pragma once
#include <stdint.h>

namespace palsgd {
namespace block {

// What an argument takes up: up to three axes (of any strides) of runs of contiguous bytes.
struct Region {
    uint64_t at, run;             // first byte; bytes of a run (0: nothing)
    uint64_t n[3], s[3];          // elements of an axis and its stride in bytes; an axis without steps has n = 1

    Region() = default;           // (not set: a call keeps two dozen of these and uses few)
    Region(const void* p, uint64_t bytes) : at(reinterpret_cast<uintptr_t>(p)), run(p ? bytes : 0), n{1, 1, 1}, s{0, 0, 0} {}
    Region& axis(int i, uint64_t count, int64_t stride_bytes)
    {
        if (count == 0) run = 0;
        if (count > 1 && stride_bytes > 0) { n[i] = count; s[i] = (uint64_t)stride_bytes; }
        return *this;
    }
    // the first byte behind the last run (no address at all if the strides lead past the last one)
    uint64_t end() const
    {
        unsigned __int128 e = (unsigned __int128)at + run;
        for (int i = 0; i < 3; ++i) if (s[i]) e += (unsigned __int128)s[i] * (n[i] - 1);
        return e > UINT64_MAX ? UINT64_MAX : (uint64_t)e;
    }
    bool same(const Region& o) const
    {
        bool eq = at == o.at && run == o.run;
        for (int i = 0; i < 3; ++i) eq = eq && n[i] == o.n[i] && s[i] == o.s[i];
        return eq;
    }
};

// Two regions share a byte where the difference of two of their runs' places lies in a window as long as the runs: a sum of
// (steps of one less steps of the other) times strides.  Axes of equal strides are one; the search takes the longest strides
// first, and only steps from which the rest can still reach the window.
struct Meeting {
    struct Steps { uint64_t s; int64_t lo, hi; } v[6];
    int n = 0;
    uint32_t left = 1u << 16;     // looked at before it gives up (and says no): interleaved layouts of unlike strides

    void add(uint64_t s, int64_t lo, int64_t hi)
    {
        if (s == 0) return;
        for (int i = 0; i < n; ++i)
            if (v[i].s == s) { v[i].lo += lo; v[i].hi += hi; return; }
        int i = n++;
        for (; i > 0 && v[i - 1].s < s; --i) v[i] = v[i - 1];
        v[i] = Steps{s, lo, hi};
    }
    // some steps of the axes from i on add up to a number in lo .. hi
    bool reach(int i, __int128 lo, __int128 hi)
    {
        if (i == n) return lo <= 0 && hi >= 0;
        __int128 rest_lo = 0, rest_hi = 0;
        for (int j = i + 1; j < n; ++j) { rest_lo += (__int128)v[j].lo * v[j].s; rest_hi += (__int128)v[j].hi * v[j].s; }
        const __int128 s = v[i].s, a = lo - rest_hi, b = hi - rest_lo;
        __int128 c = a >= 0 ? (a + s - 1) / s : -(-a / s), last = b >= 0 ? b / s : -((-b + s - 1) / s);
        if (c < v[i].lo) c = v[i].lo;
        if (last > v[i].hi) last = v[i].hi;
        for (; c <= last && left; ++c) {
            --left;
            if (reach(i + 1, lo - c * s, hi - c * s)) return true;
        }
        return false;
    }
};

// (of regions whose spans from the first byte to the last overlap)
inline bool meet(const Region& a, const Region& b)
{
    Meeting m;
    for (int i = 0; i < 3; ++i) m.add(a.s[i], 0, (int64_t)a.n[i] - 1);
    for (int i = 0; i < 3; ++i) m.add(b.s[i], 1 - (int64_t)b.n[i], 0);
    const __int128 d = (__int128)b.at - a.at;
    return m.reach(0, d - (__int128)a.run + 1, d + (__int128)b.run - 1);
}

// The arguments of a call: those without a byte are left out.
struct Regions {
    struct Entry { Region r; uint64_t end; int own[2]; } in[16], out[8];
    int n_in = 0, n_out = 0;
    int reads(const Region& r)
    {
        if (r.run == 0) return -1;
        in[n_in] = Entry{r, r.end(), {-1, -1}};
        return n_in++;
    }
    // own: inputs that it may be exactly
    void writes(const Region& r, int own_a = -1, int own_b = -1)
    {
        if (r.run) out[n_out++] = Entry{r, r.end(), {own_a, own_b}};
    }
    bool clash() const
    {
        auto meets = [](const Entry& a, const Entry& b) { return a.r.at < b.end && b.r.at < a.end && meet(a.r, b.r); };
        for (int i = 0; i < n_out; ++i) {
            for (int j = i + 1; j < n_out; ++j) if (meets(out[i], out[j])) return true;
            for (int j = 0; j < n_in; ++j)
                if (meets(out[i], in[j]) && !((j == out[i].own[0] || j == out[i].own[1]) && out[i].r.same(in[j].r))) return true;
        }
        return false;
    }
};

}  // namespace block
}  // namespace palsgd
