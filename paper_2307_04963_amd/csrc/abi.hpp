// Error reporting shared by the C entry points: the calling thread's last
// message, and the wrapper that lets no exception out.
#pragma once

#include <new>
#include <string>

#include "plan.hpp"

namespace dycl {

// stores the thread's message; returns the code
int fail(int code, const std::string& msg);

template <class F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const WeightsError& e) {
    return fail(DYCL_E_WEIGHTS, e.what());
  } catch (const SpecError& e) {
    return fail(DYCL_E_SPEC, e.what());
  } catch (const OomError& e) {
    return fail(DYCL_E_OOM, e.what());
  } catch (const HipError& e) {
    return fail(DYCL_E_HIP, e.what());
  } catch (const std::bad_alloc&) {
    return fail(DYCL_E_OOM, "host allocation failed");
  } catch (const std::exception& e) {
    return fail(DYCL_E_INVALID, e.what());
  } catch (...) {
    return fail(DYCL_E_INVALID, "unknown failure");
  }
}

}  // namespace dycl
