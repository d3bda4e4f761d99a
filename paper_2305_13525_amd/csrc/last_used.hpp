// What was worked out for the last sizes that were asked for.  Plain C++: of the host code only.
#pragma once
#include <stdint.h>

namespace axo {

// Up to N values by the three sizes that each belongs to; the one that was made longest ago makes room.  All N are looked at: a slot computed from the
// sizes would be the same one for most layers of a model, whose sizes are multiples of 128.  For one thread.
template <typename T, int N>
class LastUsed {
    int64_t sizes[N][3];
    T values[N];
    int used = 0, next = 0;

  public:
    // The value for (a, b, c), made by make() if it is not here.  Until N others have been made it stays where it is.  If make() throws nothing changes.
    template <typename F>
    const T& get(int64_t a, int64_t b, int64_t c, F make) {
        for (int i = 0; i < used; ++i)
            if (sizes[i][0] == a && sizes[i][1] == b && sizes[i][2] == c) return values[i];
        T made = make();
        const int at = next;
        values[at] = made;
        sizes[at][0] = a;
        sizes[at][1] = b;
        sizes[at][2] = c;
        next = (next + 1) % N;
        if (used < N) ++used;
        return values[at];
    }
};

}  // namespace axo
