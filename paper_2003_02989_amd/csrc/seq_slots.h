// seq_slots.h -- what segments of a scan publish for one another, and how a state
// is put together from it; plain arithmetic, the same on the host and the device.
#pragma once
#include <cstdint>
#include <cstring>

#ifdef __HIPCC__
#define TQ_HD __host__ __device__ __forceinline__
#else
#define TQ_HD inline
#endif

namespace tq {

// A pair (A, B), A >= 0, or a state (-0, h), as one 64-bit word; all ones: not
// published yet.
using Slot = unsigned long long;
constexpr Slot kEmpty = ~(Slot)0;
constexpr uint32_t kState = 0x80000000u, kNan = 0x7fc00000u;

struct SlotPair {
    uint32_t a;  // bits of A, or kState
    float b;
};

TQ_HD uint32_t slot_bits(float f)
{
    uint32_t u;
    memcpy(&u, &f, sizeof u);
    return u;
}

TQ_HD float slot_float(uint32_t u)
{
    float f;
    memcpy(&f, &u, sizeof f);
    return f;
}

TQ_HD Slot state_slot(float h) { return (Slot)kState << 32 | slot_bits(h); }
// A NaN A has one form, which is not kEmpty's.
TQ_HD Slot pair_slot(float a, float b) { return (Slot)(a == a ? slot_bits(a) : kNan) << 32 | slot_bits(b); }

// Whether a wait for what is in a slot, or (`state`) for a state in it, is over.
TQ_HD bool slot_ready(Slot v, bool state) { return v != kEmpty && (!state || (uint32_t)(v >> 32) == kState); }

// What a wait that saw `v` last gives.  One that ran out gives a state of NaN: what
// comes after it, in every output, shows that it is not known.
TQ_HD SlotPair slot_value(Slot v, bool state)
{
    if (!slot_ready(v, state)) return SlotPair{kState, slot_float(kNan)};
    return SlotPair{(uint32_t)(v >> 32), slot_float((uint32_t)v)};
}

// The state after a segment from that before it: a state starts anew.
TQ_HD float slot_step(SlotPair q, float h)
{
    return q.a == kState ? q.b : __builtin_fmaf(slot_float(q.a), h, q.b);
}

} // namespace tq
