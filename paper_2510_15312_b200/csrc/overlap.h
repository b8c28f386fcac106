// Whether two strided arrays share memory.  Host code.
#pragma once
#include <stdint.h>

namespace sdv {

// Runs of `run` bytes, up to three dimensions of them `step` bytes apart; null: an array that is not there.
struct Area {
    const void* p;
    long long run;
    struct { long long n, step; } dim[3];
    // First byte and the one behind the last; all of memory where a stride leads out of it.
    void range(uintptr_t& lo, uintptr_t& hi) const {
        lo = (uintptr_t)p;
        hi = lo + (uintptr_t)run;
        bool far = hi < lo;
        for (const auto& d : dim) {
            long long by;
            if (d.n <= 1) continue;
            if (__builtin_mul_overflow(d.n - 1, d.step, &by)) far = true;
            else if (by < 0) far |= __builtin_sub_overflow(lo, (uintptr_t)0 - (uintptr_t)by, &lo);
            else far |= __builtin_add_overflow(hi, (uintptr_t)by, &hi);
        }
        if (far) {
            lo = 0;
            hi = ~(uintptr_t)0;
        }
    }
};
inline Area area(const void* p, long long run, long long n0 = 1, long long step0 = 0, long long n1 = 1, long long step1 = 0, long long n2 = 1, long long step2 = 0) {
    return Area{p, run, {{n0, step0}, {n1, step1}, {n2, step2}}};
}

// Two arrays meet where the difference of their starts is a sum of steps, of one array forwards and of the other backwards, up to less than a run.  Steps are gone
// through from the largest down; as long as they are nested (rows of heads of elements), each leaves a few candidates.
class Overlap {
public:
    bool operator()(const Area& a, const Area& b) {
        if (!a.p || !b.p) return false;
        uintptr_t a0, a1, b0, b1;
        a.range(a0, a1);
        b.range(b0, b1);
        if (a1 <= b0 || b1 <= a0) return false;   // as good as always
        n_ = 0;
        budget_ = 4096;
        if (!add(a, -1) || !add(b, 1)) return false;
        const wide delta = (wide)(intptr_t)b.p - (wide)(intptr_t)a.p;
        return reaches(0, -delta - b.run, -delta + a.run) && budget_ >= 0;
    }

private:
    typedef __int128 wide;
    struct { wide step, lo, hi; } d_[6];   // multiples lo .. hi of a step, steps descending
    int n_, budget_;

    bool add(const Area& x, int sign) {   // false: an array without elements
        if (x.run <= 0) return false;
        for (const auto& e : x.dim) {
            if (e.n <= 0) return false;
            if (e.n == 1 || e.step == 0) continue;
            const wide step = e.step < 0 ? -(wide)e.step : e.step, far = (e.step < 0 ? -sign : sign) * (wide)(e.n - 1), lo = far < 0 ? far : 0, hi = far < 0 ? 0 : far;
            int at = 0;
            while (at < n_ && d_[at].step > step) ++at;
            if (at < n_ && d_[at].step == step) {
                d_[at].lo += lo;
                d_[at].hi += hi;
                continue;
            }
            for (int k = n_++; k > at; --k) d_[k] = d_[k - 1];
            d_[at].step = step;
            d_[at].lo = lo;
            d_[at].hi = hi;
        }
        return true;
    }
    static wide down(wide x, wide by) { return x >= 0 ? x / by : -((-x + by - 1) / by); }
    // Whether steps i and on add up to something between `from` and `to` (both excluded).  Where that takes too many candidates it is left open: no.
    bool reaches(int i, wide from, wide to) {
        if (i == n_) return from < 0 && 0 < to;
        wide least = 0, most = 0;   // of the steps behind this one
        for (int k = i + 1; k < n_; ++k) {
            least += d_[k].lo * d_[k].step;
            most += d_[k].hi * d_[k].step;
        }
        wide x = down(from - most, d_[i].step) + 1, last = down(to - least - 1, d_[i].step);
        if (x < d_[i].lo) x = d_[i].lo;
        if (last > d_[i].hi) last = d_[i].hi;
        for (; x <= last; ++x) {
            if (--budget_ < 0) return false;
            if (reaches(i + 1, from - x * d_[i].step, to - x * d_[i].step)) return true;
        }
        return false;
    }
};

}  // namespace sdv
