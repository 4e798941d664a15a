// What every extern "C" function of the library shares: failures leave as exceptions inside, as codes outside.
#pragma once
#include <new>
#include <string>

#include "engine.h"

// error text of the calls that have no context
inline thread_local std::string g_init_error;

[[noreturn]] inline void fail(int code, const std::string& msg) { throw ApiError{code, msg}; }

template <typename F>
int guarded(rollout_ctx* ctx, F&& body) {
  std::string* err = ctx ? &ctx->err : &g_init_error;
  try {
    body();
    return ROLLOUT_OK;
  } catch (const ApiError& e) {
    *err = e.msg;
    return e.code;
  } catch (const HipError& e) {
    *err = std::string("HIP error ") + hipGetErrorString(e.code) + " in " + e.expr + " (" + e.file + ":" +
           std::to_string(e.line) + ")";
    return ROLLOUT_E_HIP;
  } catch (const std::bad_alloc&) {
    *err = "host allocation failed";
    return ROLLOUT_E_NOMEM;
  } catch (...) {
    *err = "unexpected internal error";
    return ROLLOUT_E_STATE;
  }
}
