// Frequencies of rotary positions in turns per position, as 64-bit fractions of a turn: host arithmetic with 64 significant bits, of integers
// alone (doubles have 53, and what a long double has depends on the host).
#pragma once
#include <cmath>
#include <cstdint>

namespace hc {

// m 2^(e - 64), m with its highest bit set, or zero
struct Extended {
  uint64_t m;
  int e;
};

inline Extended extended(double x) {  // exact; x finite and not negative
  int e;
  return {static_cast<uint64_t>(std::frexp(x, &e) * 0x1p64), e};
}

inline Extended product(Extended a, Extended b) {  // rounded to nearest
  const unsigned __int128 p = static_cast<unsigned __int128>(a.m) * b.m;
  const int drop = 63 + static_cast<int>(p >> 127);
  const unsigned __int128 r = (p + (static_cast<unsigned __int128>(1) << (drop - 1))) >> drop;
  const int e = a.e + b.e + drop - 64;
  return r >> 64 ? Extended{uint64_t(1) << 63, e + 1} : Extended{static_cast<uint64_t>(r), e};
}

// theta^(-1/n), theta > 0, n >= 1, within 3 * 2^-64 of itself.  One Newton step on the double r nearest to it: with theta r^n = 1 + d the root is
// r (1 - d / n), but for the square of d.  (Its power in x87 arithmetic took 100 ns.)
inline Extended inverse_root(double theta, int n) {
  const Extended r = extended(std::pow(theta, -1.0 / n));
  Extended one = extended(theta), power = r;
  for (int k = n; k; k >>= 1) {
    if (k & 1) one = product(one, power);
    power = product(power, power);
  }
  // d in units of 2^-64: `one` lies at or above 1 (e = 1) or below (e = 0)
  const double d = static_cast<double>(static_cast<int64_t>(one.e == 1 ? one.m << 1 : one.m));
  const __int128 m = static_cast<__int128>(r.m) - static_cast<__int128>(static_cast<double>(r.m) * 0x1p-64 * d / n);
  if (m >> 64) return {uint64_t(1) << 63, r.e + 1};
  if (!(m >> 63)) return {static_cast<uint64_t>(m) << 1, r.e - 1};
  return {static_cast<uint64_t>(m), r.e};
}

// What is left of x turns without whole ones, in 2^-64 turns.
inline uint64_t fraction_of_turn(Extended x) {
  if (x.e >= 64 || x.e <= -64) return 0;
  return x.e > 0 ? x.m << x.e : x.m >> -x.e;
}

constexpr Extended TURNS_PER_RADIAN = {0xa2f9836e4e44152aull, -2};

}  // namespace hc
